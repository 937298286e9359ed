// Log probabilities of given classes, entropy and top alternatives of rows of margins, and their gradient.
//
// A row z of C margins (a class that is not allowed counts as -inf, the reference class as 0) has, as in eq. (8), (9),
//   M = max_c z_c,  s = sum_c e^{z_c - M},  t = sum_c e^{z_c - M} (z_c - M) <= 0,
//   log p_y = (z_y - M) - log s,  H = -sum_c p_c log p_c = log s - t / s  (two terms >= 0: nothing cancels),
// and log s in [0, log C] is kept apart from M, so that log p_y carries no rounding of a large log-sum-exp.  One pass over
// the row: every lane keeps (M, s, t) of what it has seen and rescales s and t when its M grows; pairs are joined the same
// way across lanes, waves and workgroups.  s is NaN exactly when a margin is NaN or +inf, and 0 exactly when no class is
// left (the largest margin contributes e^0 = 1).  A lane may let its M lag a little behind (Gather), and takes back what its t
// then holds too much before it is joined.  All of it in fp32 for fp32, fp16 and bf16 margins, in fp64 for fp64.
//
// What bounds it: on many long rows the vector units (11 instructions a margin) as much as memory (8192 x 65536 bf16, one label: 181
// to 187 us in a queue of passes, 5.7 to 5.9 TB/s; single launches in a trace 180 to 208).  Where a row is one workgroup's, the
// vector units 60 % of the time and the first loads and last joins around that; launch and latency on single rows (32000 fp32, five
// alternatives: 9.5 us a call, as the kernel alone).
#include "ssn_internal.h"
#include "ssn_math.h"

#include <type_traits>

namespace ssn {

namespace {

constexpr int WAVE = 64;
constexpr int NARROW_PER_LANE = 8;      // margins per lane of the narrow form

template <typename T> struct Acc { typedef float type; };
template <> struct Acc<double> { typedef double type; };

// x where m is -1, -inf where m is 0
__device__ __forceinline__ float keep_if(float x, int m)
{
    return __uint_as_float((__float_as_uint(x) & (uint32_t)m) | (0xff800000u & ~(uint32_t)m));
}
__device__ __forceinline__ double keep_if(double x, int m)
{
    const long long b = __double_as_longlong(x);
    const uint32_t lo = (uint32_t)b & (uint32_t)m, hi = ((uint32_t)(b >> 32) & (uint32_t)m) | (0xfff00000u & ~(uint32_t)m);
    return __longlong_as_double(((long long)hi << 32) | lo);
}

// 16 bytes of margins at an address aligned to an element only
typedef uint32_t Raw __attribute__((ext_vector_type(4)));
typedef Raw RawAt2 __attribute__((aligned(2)));
typedef Raw RawAt4 __attribute__((aligned(4)));
template <typename T> struct Vec {
    static constexpr int E = 16 / sizeof(T);
    typedef typename std::conditional<sizeof(T) == 2, RawAt2, RawAt4>::type RawAt;
    static __device__ __forceinline__ Raw load(const T *p) { return *(const RawAt *)p; }
    // past the caches, which a gradient of any size worth a kernel outgrows: 8192 x 65536 bf16 373 -> 355 us, 1021 x 32003 fp32 55 -> 51 us
    static __device__ __forceinline__ void store(T *p, Raw v) { __builtin_nontemporal_store(v, (RawAt *)p); }
};

__device__ __forceinline__ void unpack(Raw r, float (&x)[4], float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void unpack(Raw r, double (&x)[2], double)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = __longlong_as_double(((long long)r[2 * i + 1] << 32) | r[2 * i]);
}
__device__ __forceinline__ void unpack(Raw r, float (&x)[8], __bf16)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(Raw r, float (&x)[8], _Float16)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r[i] & 0xffffu));
        x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r[i] >> 16));
    }
}
__device__ __forceinline__ Raw pack(const float (&x)[4], float)
{
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
    return r;
}
__device__ __forceinline__ Raw pack(const double (&x)[2], double)
{
    Raw r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = (uint32_t)__double_as_longlong(x[i]);
        r[2 * i + 1] = (uint32_t)(__double_as_longlong(x[i]) >> 32);
    }
    return r;
}
// one rounding, to nearest, of the finished fp32 value
template <typename T> __device__ __forceinline__ Raw pack(const float (&x)[8], T)
{
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i]) | ((uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i + 1]) << 16);
    return r;
}

__device__ __forceinline__ float lowest(float) { return -__FLT_MAX__; }
__device__ __forceinline__ double lowest(double) { return -__DBL_MAX__; }
__device__ __forceinline__ float minus_inf(float) { return -__builtin_inff(); }
__device__ __forceinline__ double minus_inf(double) { return -__builtin_inf(); }
// -inf that the compiler does not know: it would keep a wave's constant of this value in a pair of scalar registers, and
// writes it there with one instruction that holds only half of the number.  Where minus_inf(double) stands below the compiler
// does not do that; the build goes through the assembler's text, which refuses it.
__device__ __forceinline__ float hidden_minus_inf(float) { return minus_inf(0.0f); }
__device__ __forceinline__ double hidden_minus_inf(double)
{
    int hi = (int)0xfff00000;
    asm volatile("" : "+v"(hi));
    return __longlong_as_double((long long)hi << 32);
}
__device__ __forceinline__ float nan_of(float) { return __builtin_nanf(""); }
__device__ __forceinline__ double nan_of(double) { return __builtin_nan(""); }

// e^d for d <= 0 and NaN.  fp32: 2^(d log2 e), one hardware instruction behind one rounded product -- a relative error of
// about |d| 2^-24, on a term that weighs e^d in its sum.
__device__ __forceinline__ float exp_term(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504f); }
__device__ __forceinline__ double exp_term(double d) { return d == d ? exp_nonpos(d, 0.0) : d; }
// the same with the product's rounding error put back, for results that are returned one by one in fp32
__device__ __forceinline__ float exp_value(float d)
{
    const float c = 1.44269504f, t = d * c;
    const float lo = fmaf(d, c, -t) + d * 1.925963033e-08f;           // log2 e = c + 1.926e-8
    const float r = __builtin_amdgcn_exp2f(t);
    return r > 0.0f ? fmaf(r, lo * 0.693147181f, r) : r;              // d = -inf: 0, and no product with lo = NaN
}
__device__ __forceinline__ double exp_value(double d) { return exp_term(d); }

__device__ __forceinline__ float log_sum(float s) { return logf(s); }
__device__ __forceinline__ double log_sum(double s) { return s == s ? log_ge1(s) : s; }

template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_or_lowest(float x)
{
    const float id = minus_inf(0.0f);
    return __uint_as_float(__builtin_amdgcn_update_dpp((int)__float_as_uint(id), (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_or_lowest(double x)
{
    const long long b = __double_as_longlong(x), id = __double_as_longlong(minus_inf(0.0));
    const int lo = __builtin_amdgcn_update_dpp((int)id, (int)b, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp((int)(id >> 32), (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double(((long long)hi << 32) | (long long)(unsigned)lo);
}
__device__ __forceinline__ float at_lane(float x, int lane)
{
    return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}
__device__ __forceinline__ double at_lane(double x, int lane)
{
    const long long b = __double_as_longlong(x);
    const unsigned lo = __builtin_amdgcn_readlane((int)b, lane);
    const int hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __longlong_as_double(((long long)hi << 32) | (long long)lo);
}
template <typename A> __device__ __forceinline__ A take_max(A a, A b) { return a > b ? a : b; }
__device__ __forceinline__ float take_max(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double take_max(double a, double b) { return fmax(a, b); }
// largest value over the wave's 64 lanes (NaN lanes do not count)
template <typename A> __device__ __forceinline__ A wave_max(A x)
{
    x = take_max(x, dpp_or_lowest<0x111, 0xf>(x));
    x = take_max(x, dpp_or_lowest<0x112, 0xf>(x));
    x = take_max(x, dpp_or_lowest<0x114, 0xf>(x));
    x = take_max(x, dpp_or_lowest<0x118, 0xf>(x));
    x = take_max(x, dpp_or_lowest<0x142, 0xa>(x));
    x = take_max(x, dpp_or_lowest<0x143, 0xc>(x));
    return at_lane(x, 63);
}
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_or_none(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_or_none(double x) { return dpp_or_zero<CTRL, ROWS>(x); }
// the sum over the wave's 64 lanes, in a fixed order
template <typename A> __device__ __forceinline__ A wave_sum(A x)
{
    x += dpp_or_none<0x111, 0xf>(x);
    x += dpp_or_none<0x112, 0xf>(x);
    x += dpp_or_none<0x114, 0xf>(x);
    x += dpp_or_none<0x118, 0xf>(x);
    x += dpp_or_none<0x142, 0xa>(x);
    x += dpp_or_none<0x143, 0xc>(x);
    return at_lane(x, 63);
}
// The value of the lane that is O apart in a group of 2 O lanes whose halves hold one value each (O = 1, 2, 4, ... in turn):
// exchanges of lanes inside rows of sixteen, through LDS beyond
template <int O> __device__ __forceinline__ int across(int x)
{
    if (O == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false);       // lanes 1 0 3 2
    if (O == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false);       // lanes 2 3 0 1
    if (O == 4) return __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false);      // halves of a row mirrored
    if (O == 8) return __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, false);      // rows mirrored
    return __shfl_xor(x, O, WAVE);
}
template <int O> __device__ __forceinline__ float across(float x) { return __uint_as_float((uint32_t)across<O>((int)__float_as_uint(x))); }
template <int O> __device__ __forceinline__ double across(double x)
{
    const long long b = __double_as_longlong(x);
    const uint32_t lo = (uint32_t)across<O>((int)b);
    return __longlong_as_double(((long long)across<O>((int)(b >> 32)) << 32) | lo);
}
// f<O>() for O = 1, 2, ..., G / 2
template <int G, int O = 1, typename F> __device__ __forceinline__ void each_step(F f)
{
    if constexpr (O < G) {
        f(std::integral_constant<int, O>());
        each_step<G, 2 * O>(f);
    }
}

// ---- the running statistics of a row ---------------------------------------------------------------------------------
template <typename A> struct Stat {
    A M, s, t;
    __device__ __forceinline__ void init() { M = lowest(A()), s = A(0), t = A(0); }
    // M grows to `top`: d <= 0 clamped where e^d is long zero, so that 0 * (-inf) never forms
    __device__ __forceinline__ void raise(A top)
    {
        const A d = take_max(M - top, A(-1e4)), c = exp_term(d);
        t = (t + s * d) * c;
        s *= c;
        M = top;
    }
    __device__ __forceinline__ void add(A z)
    {
        const A d = z - M, e = exp_term(d);
        s += e;
        t = fma(e, take_max(d, A(-1e4)), t);
    }
    __device__ __forceinline__ void join_wave()
    {
        raise(wave_max(M));
        s = wave_sum(s);
        t = wave_sum(t);
    }
};

// What a lane gathers on its way over a long row; done() turns it into a Stat with M = the largest margin met.
// fp64: the Stat itself.
template <typename A> struct Gather {
    Stat<A> q;
    A mx;                               // the largest margin, -inf: none
    __device__ __forceinline__ void init() { q.init(), mx = minus_inf(A()); }
    template <int E> __device__ __forceinline__ void take(const A (&x)[E], A top)
    {
        mx = take_max(mx, top);
        q.raise(take_max(q.M, top));
#pragma unroll
        for (int e = 0; e < E; ++e) q.add(x[e]);
    }
    __device__ __forceinline__ Stat<A> done() const { return q; }
};
// fp32: a margin costs a fused multiply-add, 2^x, an addition, a clamp and a fused multiply-add; the kernel is as much bound
// by these as by memory.  s and t are kept relative to a power of two: s = sum 2^(c z - M2), t = sum 2^(c z - M2) (c z - M2)
// with c = log2 e rounded and M2 = c R rounded, both exactly what the multiply-add uses, so that the rounding of M2 is known
// (r = c R - M2) and taken out at the end.  R follows the largest margin when it falls more than LAG behind.  What t holds too
// much and done() takes back is at most LAG s, and the heaviest terms are rescaled by no more than e^-LAG: a wider lag saves
// rescalings and costs a confident row its last bits (a best class behind margins 3 to 13 below it in its lane, 256 x 65536:
// entropy off by 8 u with a lag of 13, u = 2^-24, root mean square, by 3 u with two or one; 8192 x 65536 bf16 179, 183 and
// 187 us).  |r| grows with R, to 0.9 at the edge below: a row whose largest margin is beyond half of that is gathered by a
// Stat instead, and in any other row a margin below -edge weighs nothing.
template <> struct Gather<float> {
    float R, M2, s, t, mx;
    static constexpr float LAG = 2.0f;
    static __device__ __forceinline__ float edge() { return 1e7f; }
    static __device__ __forceinline__ float c() { return 1.44269504f; }
    __device__ __forceinline__ void init()
    {
        R = -edge(), M2 = -edge() * c();
        s = t = 0.0f;
        mx = minus_inf(0.0f);
    }
    template <int E> __device__ __forceinline__ void take(const float (&x)[E], float top)
    {
#pragma clang fp contract(off)          // M2 - m2 below takes m2 as it is kept, rounded
        mx = fmaxf(mx, top);
        if (__ballot(top - R > LAG)) {
            const float to = fmaxf(R, top), m2 = to * c(), d = fmaxf(M2 - m2, -1e4f), f = __builtin_amdgcn_exp2f(d);
            t = (t + s * d) * f;
            s *= f;
            R = to, M2 = m2;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = fmaf(x[e], c(), -M2), ex = __builtin_amdgcn_exp2f(d);
            s += ex;
            t = fmaf(ex, fmaxf(d, -1e4f), t);
        }
    }
    __device__ __forceinline__ Stat<float> done() const
    {
        const float r = fmaf(c(), R, -M2), f = __builtin_amdgcn_exp2f(-r);
        Stat<float> q;
        q.M = R, q.s = s * f, q.t = (t - r * s) * f * (1.0f / c());
        if (s == 0.0f) q.init();
        else if (mx > R) q.raise(mx);
        return q;
    }
};
// whether a row with this largest margin is out of a Gather's reach; fp16 margins never are
template <typename T> __device__ __forceinline__ bool beyond(float top) { return sizeof(T) == 4 || std::is_same<T, __bf16>::value ? !(fabsf(top) < 5e6f) && top != minus_inf(0.0f) : false; }
template <typename T> __device__ __forceinline__ bool beyond(double) { return false; }

// One row's answer.  s == 0: no class is left; s != s: the row holds NaN or +inf at an allowed class.  Any other row has s >= 1,
// but where a Gather's reference is a power of two its largest margin's term is two rounded factors and may miss 1 by their
// error: no log probability is above zero, and no entropy below.
template <typename A> struct Answer {
    A M, L, s, t;
    __device__ __forceinline__ Answer(const Stat<A> &q) : M(q.M), s(q.s), t(q.t)
    {
        if (s > A(0) && s < A(1)) s = A(1);
        L = s == A(0) ? A(0) : log_sum(s);
    }
    __device__ __forceinline__ A maxpart() const { return s == A(0) ? minus_inf(A()) : s == s ? M : s; }
    __device__ __forceinline__ A logpart() const { return L; }
    __device__ __forceinline__ A entropy() const
    {
        const A h = s == A(0) ? A(0) : L - t / s;
        return h < A(0) ? A(0) : h;                                    // NaN stays
    }
    __device__ __forceinline__ A logp(A z) const
    {
        if (!(s == s)) return s;
        return s == A(0) || z == minus_inf(A()) ? minus_inf(A()) : (z - M) - L;
    }
};

__device__ __forceinline__ bool allowed_bit(const uint32_t *mask, int64_t c) { return (mask[c >> 5] >> (c & 31)) & 1u; }

// ---- a sorted list of alternatives: lane i < k of the wave holds the i-th best (value, class) seen, -inf where there is none --------
template <typename A> struct Best {
    A v;
    int id;
    A least;                            // the k-th best value: what does not exceed it is not taken
    __device__ __forceinline__ void init() { v = least = hidden_minus_inf(A()), id = -1; }
    // value m of class c goes behind the values >= m: classes come in ascending order, so a tie stays with the lower one
    __device__ __forceinline__ void insert(A m, int c, int lane, int k)
    {
        const int at = __popcll(__ballot(v >= m));
        const A pv = __shfl_up(v, 1, WAVE);
        const int pid = __shfl_up(id, 1, WAVE);
        if (lane > at && lane < k) v = pv, id = pid;
        if (lane == at) v = m, id = c;
        least = at_lane(v, k - 1);
    }
    // E consecutive classes per lane from `c`, lanes ascending: the largest one first, until none is above the k-th best
    template <int E> __device__ __forceinline__ void take(const A (&z)[E], int c, int lane, int k)
    {
        A lm = z[0];
#pragma unroll
        for (int e = 1; e < E; ++e) lm = take_max(lm, z[e]);
        if (!__ballot(lm > least)) return;
        A x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = z[e];
        do {
            const A m = wave_max(lm);
            const int who = __ffsll((unsigned long long)__ballot(lm == m)) - 1;
            int sel = 0;
#pragma unroll
            for (int e = E - 1; e >= 0; --e) sel = x[e] == m ? e : sel;
            const int cls = __builtin_amdgcn_readlane(c + sel, who);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (lane == who && e == sel) ? minus_inf(A()) : x[e];
            lm = x[0];
#pragma unroll
            for (int e = 1; e < E; ++e) lm = take_max(lm, x[e]);
            insert(m, cls, lane, k);
        } while (__ballot(lm > least));
    }
};

// The k best of N candidates in LDS by counting, for each, the better ones (a tie: the lower class): slot[rank] = candidate.
// Called by all `threads` of a workgroup between barriers; slots that no candidate takes keep what they hold.  Sixteen lanes
// share a candidate, so that forty of them wait for LDS three times and not forty.
template <typename A>
__device__ __forceinline__ void rank_candidates(const A *val, const int *id, int N, int k, int threads, A *slot_v, int *slot_id)
{
    const int l = threadIdx.x & 15;
    for (int i = threadIdx.x >> 4; i < N; i += threads >> 4) {
        const A v = val[i];
        const int c = id[i];
        int rank = 0;
        for (int j = l; j < N; j += 16) {
            const A o = val[j];
            rank += (int)(o > v) | ((int)(o == v) & (int)(id[j] < c));
        }
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x128, 0xf, 0xf, false);          // rotations inside a row of 16 lanes
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x124, 0xf, 0xf, false);
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x122, 0xf, 0xf, false);
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x121, 0xf, 0xf, false);
        if (l == 0 && rank < k) slot_v[rank] = v, slot_id[rank] = c;
    }
}

// A value that at least c of the wave's 64 lanes reach (c >= 1), as large as it comes cheaply; -inf where fewer hold more than
// that.  Up to 24: the c-th largest, one wave maximum after the other.  Beyond: the smallest of the maxima of 32 pairs, or of all.
template <typename A> __device__ __forceinline__ A reached_by(A v, int c)
{
    if (c <= 24) {
        A m;
        for (;;) {
            m = wave_max(v);
            const unsigned long long b = __ballot(v == m);
            c -= __popcll(b);
            if (c <= 0 || m == minus_inf(A())) return m;
            v = v == m ? minus_inf(A()) : v;
        }
    }
    if (c <= 32) v = take_max(v, __shfl_xor(v, 1, WAVE));
    return -wave_max(-v);
}
// the q-th largest of `count` <= 64 values in LDS, by all lanes of a wave; -inf where fewer are more than that
template <int COUNT, typename A> __device__ __forceinline__ A kth_of(const A *vals, int q, int lane)
{
    const A v = lane < COUNT ? vals[lane] : minus_inf(A());
    int ge = 0;                                                        // how many reach this lane's value
#pragma unroll
    for (int j = 0; j < COUNT; ++j) ge += vals[j] >= v ? 1 : 0;
    return wave_max(ge >= q ? v : minus_inf(A()));
}

template <typename T> __device__ __forceinline__ typename Acc<T>::type margin_of(const LogprobsArgs &a, int64_t row, int64_t c)
{
    typedef typename Acc<T>::type A;
    if (a.allowed && !allowed_bit(a.allowed + row * a.ld_allowed, c)) return minus_inf(A());
    if (c >= a.width) return A(0);                                     // the reference class
    return (A)((const T *)a.Z)[row * a.ldz + c];
}

// the outputs of one row by one wave: zy is the margin of given class `lane` (lanes < m), alt that of alternative `lane`
template <typename T, bool TOP>
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int64_t row, int lane, const Stat<typename Acc<T>::type> &q,
                                          int y, typename Acc<T>::type zy, typename Acc<T>::type alt, int alt_id)
{
    typedef typename Acc<T>::type A;
    const Answer<A> w(q);
    if (lane == 0) {
        if (a.maxpart) ((A *)a.maxpart)[row] = w.maxpart();
        if (a.logpart) ((A *)a.logpart)[row] = w.logpart();
        if (a.entropy) ((A *)a.entropy)[row] = w.entropy();
    }
    if (lane < a.m) ((A *)a.logp)[row * a.m + lane] = y < 0 ? A(0) : y >= a.C ? nan_of(A()) : w.logp(zy);
    if (TOP && lane < a.k) {
        a.top_ids[row * a.k + lane] = q.s == q.s ? alt_id : -1;
        ((A *)a.top_logp)[row * a.k + lane] = w.logp(alt);
    }
}

// ---- rows of many classes: WAVES waves share a row, or one of `parts` stretches of it ---------------------------------
// Each wave walks a stretch of its own, AHEAD loads of 16 bytes per lane in flight.
//
// Alternatives: every lane knows the largest margin it has met.  If c lanes of each of q waves hold at least tau and c q >= k,
// no alternative is below tau: tau is the q-th largest over the waves of their c-th largest lane maximum, with c = ceil(k /
// waves) and q = ceil(k / c).  Only lanes whose maximum reaches tau read their margins again and put those >= tau
// into LDS (a little more than k on ordinary rows), where they are ranked.  More than CAND of them (rows full of ties, or
// whose large margins sit in few lanes): the waves go over their stretches again, each keeping a sorted list.
template <typename T> struct Stretch {
    typedef typename Acc<T>::type A;
    static constexpr int E = Vec<T>::E, STEP = WAVE * E;
    const T *z;
    const uint32_t *mask;
    int64_t first, end;
    // the 16 bytes of column c1 + lane E and the word with their bits, where the wave's step from c1 is `whole` inside the
    // row, and where it reaches beyond the end; nothing here waits for what is loaded
    __device__ __forceinline__ void load(int64_t c1, int lane, bool whole, Raw &raw, uint32_t &word) const
    {
        word = 0;
        if (whole) {
            raw = Vec<T>::load(z + c1 + lane * E);
            if (mask) word = (mask + (c1 >> 5))[lane * E >> 5];
            return;
        }
        load_any(c1 + lane * E, raw, word);
    }
    __device__ __forceinline__ void load_any(int64_t c, Raw &raw, uint32_t &word) const
    {
        raw = Raw{0, 0, 0, 0};
        word = 0;
        if (c + E <= end) {
            raw = Vec<T>::load(z + c);
        } else if (c < end) {                                          // the row's last, partial vector
            T tail[E];
#pragma unroll
            for (int e = 0; e < E; ++e) tail[e] = z[c + e < end ? c + e : end - 1];
            raw = __builtin_bit_cast(Raw, tail);
        }
        if (mask && c < end) word = mask[c >> 5];
    }
    // their margins, -inf where nothing takes part
    __device__ __forceinline__ void get(int64_t c, const Raw &raw, uint32_t word, bool whole, A (&x)[E]) const
    {
        unpack(raw, x, T());
        if (mask || !whole) {
            uint32_t bits = mask ? word >> (c & 31) : (1u << E) - 1;
            if (!whole) bits = c >= end ? 0 : c + E > end ? bits & ((1u << (int)(end - c)) - 1) : bits;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = keep_if(x[e], (int)(bits << (31 - e)) >> 31);
        }
    }
};

constexpr int CAND = 1024;

template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES *WAVE) void logprobs_wide_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    typedef Stretch<T> S;
    constexpr int E = S::E, STEP = S::STEP, AHEAD = sizeof(T) == 8 ? 2 : 4;
    static_assert(WAVES * WAVE <= CAND, "a sorted list of every wave fits");
    __shared__ A sh_stat[WAVES][3], sh_kth[WAVES];
    __shared__ A sh_val[TOP ? CAND : 1], sh_slot[TOP ? WAVE : 1];
    __shared__ int sh_id[TOP ? CAND : 1], sh_slot_id[TOP ? WAVE : 1], sh_count;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int part = blockIdx.x;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        S in;
        in.z = (const T *)a.Z + row * a.ldz;
        in.mask = a.allowed ? a.allowed + row * a.ld_allowed : nullptr;
        in.first = ((int64_t)part * WAVES + wave) * a.per_wave;
        in.end = in.first + a.per_wave < a.width ? in.first + a.per_wave : a.width;
        // given classes: their margins are on the way while the row is read
        int y = -1;
        A zy = A(0);
        if (a.parts == 1 && wave == 0 && lane < a.m) {
            y = a.labels[row * a.m + lane];
            if (y >= 0 && y < a.C) zy = margin_of<T>(a, row, y);
        }
        Gather<A> acc;
        acc.init();
        // the lane's second and third largest maximum of a vector (acc.mx is the largest), and the steps of the first two
        A v2 = minus_inf(A()), v3 = minus_inf(A());
        int at1 = 0, at2 = 0;
        Raw raw[AHEAD];
        uint32_t word[AHEAD];
        for (int64_t c1 = in.first; c1 < in.end; c1 += AHEAD * STEP) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) in.load(c1 + u * STEP, lane, c1 + (u + 1) * STEP <= in.end, raw[u], word[u]);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (c1 + u * STEP >= in.end) break;
                A x[E];
                in.get(c1 + u * STEP + lane * E, raw[u], word[u], c1 + (u + 1) * STEP <= in.end, x);
                A top = x[0];
#pragma unroll
                for (int e = 1; e < E; ++e) top = take_max(top, x[e]);
                if (TOP) {
                    const bool over1 = top > acc.mx, over2 = top > v2;
                    const int here = (int)(c1 + u * STEP - in.first);
                    v3 = over2 ? v2 : take_max(v3, top);
                    at2 = over1 ? at1 : over2 ? here : at2;
                    v2 = over1 ? acc.mx : over2 ? top : v2;
                    at1 = over1 ? here : at1;
                }
                acc.take(x, top);
            }
        }
        const A v1 = acc.mx;
        Stat<A> q = acc.done();
        if constexpr (sizeof(T) == 4 || std::is_same<T, __bf16>::value) {
            A top = wave_max(v1);
            if (WAVES > 1) {
                if (lane == 0) sh_kth[wave] = top;
                __syncthreads();
                top = wave_max(lane < WAVES ? sh_kth[lane] : minus_inf(A()));
                __syncthreads();
            }
            if (beyond<T>(top)) {
                q.init();
                for (int64_t c1 = in.first; c1 < in.end; c1 += STEP) {
                    Raw far;
                    uint32_t bits;
                    A x[E];
                    in.load_any(c1 + lane * E, far, bits);
                    in.get(c1 + lane * E, far, bits, false, x);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        q.raise(take_max(q.M, x[e]));
                        q.add(x[e]);
                    }
                }
            }
        }
        // the reference class, behind all others, is lane 0's of the last wave
        const bool with_ref = a.reference && part == a.parts - 1 && wave == WAVES - 1 && lane == 0 &&
                              (!in.mask || allowed_bit(in.mask, a.width));
        if (with_ref) {
            q.raise(take_max(q.M, A(0)));
            q.add(A(0));
        }
        const int c = (a.k + WAVES - 1) / WAVES;
        A kth = minus_inf(A());
        if (TOP) {
            kth = reached_by(with_ref ? take_max(v1, A(0)) : v1, c);
            if (threadIdx.x == 0) sh_count = 0;
            if (threadIdx.x < WAVE) sh_slot[lane] = minus_inf(A()), sh_slot_id[lane] = -1;
        }
        q.join_wave();
        if (lane == 0) sh_stat[wave][0] = q.M, sh_stat[wave][1] = q.s, sh_stat[wave][2] = q.t, sh_kth[wave] = kth;
        __syncthreads();
        if (TOP) {
            A tau = kth;
            if (WAVES > 1) tau = kth_of<WAVES>(sh_kth, (a.k + c - 1) / c, lane);
            tau = take_max(tau, lowest(A()));                          // -inf is no alternative
            auto put = [&](int64_t col, const A (&x)[E]) {
                uint32_t hit = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) hit |= (uint32_t)(x[e] >= tau) << e;
                if (!hit) return;
                int at = atomicAdd(&sh_count, __popc(hit));
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if ((hit >> e) & 1u) {
                        if (at < CAND) sh_val[at] = x[e], sh_id[at] = (int)(col + e);
                        ++at;
                    }
            };
            if (v1 >= tau) {
                Raw r1, r2;
                uint32_t w1, w2;
                A x[E];
                if (v3 < tau) {                                        // all of the lane's are in one vector or two
                    const int64_t col = in.first + lane * E;
                    if (a.per_wave <= AHEAD * STEP) {                  // and those are still here
                        r1 = r2 = raw[0], w1 = w2 = word[0];
#pragma unroll
                        for (int u = 1; u < AHEAD; ++u) {
                            if (at1 == u * STEP) r1 = raw[u], w1 = word[u];
                            if (at2 == u * STEP) r2 = raw[u], w2 = word[u];
                        }
                    } else {
                        in.load_any(col + at1, r1, w1);
                        if (v2 >= tau) in.load_any(col + at2, r2, w2);
                    }
                    in.get(col + at1, r1, w1, false, x);
                    put(col + at1, x);
                    if (v2 >= tau) {
                        in.get(col + at2, r2, w2, false, x);
                        put(col + at2, x);
                    }
                } else {
                    for (int64_t col = in.first + lane * E; col < in.end; col += STEP) {
                        in.load_any(col, r1, w1);
                        in.get(col, r1, w1, false, x);
                        put(col, x);
                    }
                }
            }
            if (with_ref && A(0) >= tau) {
                const int at = atomicAdd(&sh_count, 1);
                if (at < CAND) sh_val[at] = A(0), sh_id[at] = (int)a.width;
            }
            __syncthreads();
            int N = sh_count;
            if (N > CAND) {
                __syncthreads();
                Best<A> best;
                best.init();
                for (int64_t c1 = in.first; c1 < in.end; c1 += STEP) {
                    Raw raw;
                    uint32_t word;
                    A x[E];
                    in.load_any(c1 + lane * E, raw, word);
                    in.get(c1 + lane * E, raw, word, false, x);
                    best.take(x, (int)(c1 + lane * E), lane, a.k);
                }
                if (__ballot(with_ref) && A(0) > best.least) best.insert(A(0), (int)a.width, lane, a.k);
                if (lane < a.k) sh_val[wave * a.k + lane] = best.v, sh_id[wave * a.k + lane] = best.id;
                N = WAVES * a.k;
                __syncthreads();
            }
            rank_candidates(sh_val, sh_id, N, a.k, WAVES * WAVE, sh_slot, sh_slot_id);
            __syncthreads();
        }
        if (wave == 0) {
            if (WAVES > 1) {
                q.init();
                if (lane < WAVES) q.M = sh_stat[lane][0], q.s = sh_stat[lane][1], q.t = sh_stat[lane][2];
                q.join_wave();
            }
            const A tv = TOP ? sh_slot[lane] : A(0);
            const int ti = TOP ? sh_slot_id[lane] : -1;
            if (a.parts == 1) {
                write_row<T, TOP>(a, row, lane, q, y, zy, tv, ti);
            } else {
                const int64_t item = row * a.parts + part;
                if (lane == 0) {
                    A *w = (A *)a.ws_stat + item * 3;
                    w[0] = q.M, w[1] = q.s, w[2] = q.t;
                }
                if (TOP && lane < a.k) ((A *)a.ws_val)[item * a.k + lane] = tv, a.ws_id[item * a.k + lane] = ti;
            }
        }
        __syncthreads();
    }
}

// The parts of a row joined, a workgroup per row.  No alternative of the row is below the k-th of any part.
template <typename T, bool TOP> __global__ __launch_bounds__(TOP ? VEC_BLOCK : WAVE) void logprobs_join_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    __shared__ A sh_val[TOP ? LOGPROBS_MAX_PARTS * WAVE : 1], sh_slot[TOP ? WAVE : 1];
    __shared__ int sh_id[TOP ? LOGPROBS_MAX_PARTS * WAVE : 1], sh_slot_id[TOP ? WAVE : 1], sh_count;
    const int lane = threadIdx.x & (WAVE - 1);
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        int y = -1;
        A zy = A(0);
        if (threadIdx.x < a.m) {
            y = a.labels[row * a.m + threadIdx.x];
            if (y >= 0 && y < a.C) zy = margin_of<T>(a, row, y);
        }
        Stat<A> q;
        q.init();
        if (lane < a.parts) {
            const A *w = (const A *)a.ws_stat + (row * a.parts + lane) * 3;
            q.M = w[0], q.s = w[1], q.t = w[2];
        }
        if (TOP) {
            const int64_t at = row * a.parts * a.k;
            const int N = a.parts * a.k;
            A kth = minus_inf(A()), v = minus_inf(A());
            int id = -1;
            if (lane < a.parts) kth = ((const A *)a.ws_val)[at + lane * a.k + a.k - 1];
            if (threadIdx.x < N) v = ((const A *)a.ws_val)[at + threadIdx.x], id = a.ws_id[at + threadIdx.x];
            if (threadIdx.x == 0) sh_count = 0;
            if (threadIdx.x < WAVE) sh_slot[lane] = minus_inf(A()), sh_slot_id[lane] = -1;
            __syncthreads();
            const A tau = wave_max(kth);
            for (int i = threadIdx.x; i < N; i += VEC_BLOCK) {
                if (i >= VEC_BLOCK) v = ((const A *)a.ws_val)[at + i], id = a.ws_id[at + i];
                if (v >= tau && v > minus_inf(A())) {
                    const int slot = atomicAdd(&sh_count, 1);
                    sh_val[slot] = v, sh_id[slot] = id;
                }
            }
            __syncthreads();
            rank_candidates(sh_val, sh_id, sh_count, a.k, VEC_BLOCK, sh_slot, sh_slot_id);
            __syncthreads();
        }
        q.join_wave();
        if (threadIdx.x < WAVE) write_row<T, TOP>(a, row, lane, q, y, zy, TOP ? sh_slot[lane] : A(0), TOP ? sh_slot_id[lane] : -1);
        if (TOP) __syncthreads();
    }
}

// ---- rows of few classes: G lanes per row, at most NARROW_PER_LANE margins each, all in registers ----------------------
template <typename T, int G> __global__ __launch_bounds__(VEC_BLOCK) void logprobs_narrow_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    constexpr int R = NARROW_PER_LANE;
    const int g = threadIdx.x & (G - 1);
    const int64_t rows = VEC_BLOCK / G;
    for (int64_t base = (int64_t)blockIdx.x * rows; base < a.n; base += (int64_t)gridDim.x * rows) {
        const int64_t row = base + threadIdx.x / G;
        const bool live = row < a.n;                                   // idle lanes stay for the exchanges below
        A x[R];
        const T *z = (const T *)a.Z + (live ? row : 0) * a.ldz + g;
        T raw[R];
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = g + r * G < a.width ? z[r * G] : (T)0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = g + r * G < a.C ? (A)raw[r] : minus_inf(A());        // 0: the reference class
        if (a.allowed) {
            const uint32_t *mask = a.allowed + (live ? row : 0) * a.ld_allowed;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (g + r * G < a.C && !allowed_bit(mask, g + r * G)) x[r] = minus_inf(A());
        }
        Stat<A> q;
        q.init();
#pragma unroll
        for (int r = 0; r < R; ++r) q.M = take_max(q.M, x[r]);
        each_step<G>([&](auto o) { q.M = take_max(q.M, across<decltype(o)::value>(q.M)); });
#pragma unroll
        for (int r = 0; r < R; ++r) q.add(x[r]);
        each_step<G>([&](auto o) {
            q.s += across<decltype(o)::value>(q.s);
            q.t += across<decltype(o)::value>(q.t);
        });
        const Answer<A> w(q);
        if (live && g == 0) {
            if (a.maxpart) ((A *)a.maxpart)[row] = w.maxpart();
            if (a.logpart) ((A *)a.logpart)[row] = w.logpart();
            if (a.entropy) ((A *)a.entropy)[row] = w.entropy();
        }
        for (int i = g; live && i < a.m; i += G) {
            const int y = a.labels[row * a.m + i];
            ((A *)a.logp)[row * a.m + i] =
                y < 0 ? A(0) : y >= a.C ? nan_of(A()) : w.logp(margin_of<T>(a, row, y));
        }
        for (int i = 0; i < a.k; ++i) {                                // the largest margin left, then the lowest class with it
            A v = x[0];
#pragma unroll
            for (int r = 1; r < R; ++r) v = take_max(v, x[r]);
            each_step<G>([&](auto o) { v = take_max(v, across<decltype(o)::value>(v)); });
            int id = -1;
#pragma unroll
            for (int r = R - 1; r >= 0; --r) id = x[r] == v ? g + r * G : id;
            id = v > minus_inf(A()) ? id : -1;
            each_step<G>([&](auto o) {
                const int oid = across<decltype(o)::value>(id);
                id = (unsigned)oid < (unsigned)id ? oid : id;
            });
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = id == g + r * G ? minus_inf(A()) : x[r];
            if (live && g == 0) {
                a.top_ids[row * a.k + i] = q.s == q.s ? id : -1;
                ((A *)a.top_logp)[row * a.k + i] = w.logp(v);
            }
        }
    }
}

// ---- gradient --------------------------------------------------------------------------------------------------------
// dz_c = sum_t g_t (1[c = y_t] - p_c) + l p_c - h p_c (log p_c + H): one product with -p_c, then the given classes' own
// terms in the order in which they are given.  A class that has no probability takes no gradient from its log probability.
template <typename A> struct RowGrad {
    A M, L, H, h, G;                    // G = sum_t g_t - l
    bool empty;
    __device__ __forceinline__ void load(const LogprobsArgs &a, int64_t row)
    {
        M = ((const A *)a.maxpart)[row];
        L = ((const A *)a.logpart)[row];
        h = a.dentropy ? ((const A *)a.dentropy)[row] : A(0);
        H = a.dentropy ? ((const A *)a.entropy)[row] : A(0);
        G = a.dlse ? -((const A *)a.dlse)[row] : A(0);
        empty = M == minus_inf(A());
    }
    __device__ __forceinline__ A at(A z) const
    {
        const A lp = (z - M) - L;
        A w = G;
        if (h != A(0)) w = fma(h, take_max(lp, A(-1e4)) + H, w);
        return -exp_value(lp) * w;
    }
    // A vector of them.  16-bit results take one multiply-add for the exponent: with k = c M rounded and r = c M - k, which is
    // exact, p = 2^(c z - k) f with f = 2^(-r - c L), a factor of the row; what is left of p's error, |c (z - M)| 2^-24, is
    // far below their rounding.  Where r is no longer small, at() does it.
    template <typename T, int E> __device__ __forceinline__ void values(A (&x)[E]) const
    {
        if constexpr (sizeof(T) == 2) {
            if (fabsf(M) < 5e6f) {
                const float c = 1.44269504f, k = M * c, r = fmaf(M, c, -k), f = __builtin_amdgcn_exp2f(-fmaf(L, c, r));
                if (h == 0.0f) {
                    const float w = -G * f;
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], c, -k)) * w;
                } else {
                    // G + h (log p + H) with log p = (d - r) / c - L
                    const float slope = -f * h * (1.0f / c), base = -f * fmaf(h, H - L - r * (1.0f / c), G);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float d = fmaf(x[e], c, -k);
                        x[e] = __builtin_amdgcn_exp2f(d) * fmaf(slope, fmaxf(d, -1e4f), base);
                    }
                }
                return;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = at(x[e]);
    }
};
// given class y's weight: none for padding and for a class without probability, NaN for an index that is no class
template <typename A> __device__ __forceinline__ A given_weight(const LogprobsArgs &a, int64_t at, int y)
{
    if (y < 0) return A(0);
    if (y >= a.C) return nan_of(A());
    return ((const A *)a.logp)[at] == minus_inf(A()) ? A(0) : ((const A *)a.dlogp)[at];
}

// WAVES waves walk a stretch of a row, GRAD_AHEAD loads of 16 bytes per thread in flight; the row's statistics and given
// classes are fetched behind the first of them.
constexpr int GRAD_AHEAD = 2;
template <typename T, int WAVES> __global__ __launch_bounds__(WAVES *WAVE) void logprobs_grad_wide_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    constexpr int E = Vec<T>::E, STEP = WAVES * WAVE * E, AHEAD = GRAD_AHEAD;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t first = (int64_t)blockIdx.x * a.per_wave, end = first + a.per_wave < a.width ? first + a.per_wave : a.width;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        Stretch<T> in;
        in.z = (const T *)a.Z + row * a.ldz;
        in.mask = a.allowed ? a.allowed + row * a.ld_allowed : nullptr;
        in.first = first, in.end = end;
        T *dz = (T *)a.dZ + row * a.lddz;
        Raw raw[AHEAD];
        uint32_t word[AHEAD];
        auto fetch = [&](int64_t c0, int u) {
            const int64_t c1 = c0 + u * STEP + wave * WAVE * E;
            in.load(c1, lane, c1 + WAVE * E <= end, raw[u], word[u]);
        };
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) fetch(first, u);
        int y = -1;
        A gy = A(0);
        if (lane < a.m) {
            y = a.labels[row * a.m + lane];
            gy = given_weight<A>(a, row * a.m + lane, y);
        }
        RowGrad<A> w;
        w.load(a, row);
        w.G += wave_sum(gy);
        for (int64_t c0 = first; c0 < end; c0 += AHEAD * STEP) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t c1 = c0 + u * STEP + wave * WAVE * E;    // the wave's columns
                if (c1 >= end) break;
                const bool whole = c1 + WAVE * E <= end;
                const int64_t c = c1 + lane * E;
                A x[E];
                unpack(raw[u], x, T());
                const uint32_t bits = in.mask ? word[u] >> (c & 31) : 0xffffffffu;
                if (c0 + AHEAD * STEP < end) fetch(c0 + AHEAD * STEP, u);
                if (w.empty) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = A(0);
                } else {
                    w.template values<T>(x);
                    if (in.mask) {
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = (bits >> e) & 1u ? x[e] : A(0);
                    }
                }
                for (unsigned long long b = __ballot(gy != A(0) && y >= c1 && y < c1 + WAVE * E); b; b &= b - 1) {
                    const int from = __ffsll(b) - 1;
                    const int64_t yy = __builtin_amdgcn_readlane(y, from);
                    const A g = at_lane(gy, from);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] += c + e == yy && ((bits >> e) & 1u) ? g : A(0);
                }
                if (whole || c + E <= end) {
                    Vec<T>::store(dz + c, pack(x, T()));
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (c + e < end) dz[c + e] = (T)x[e];
                }
            }
        }
    }
}

template <typename T, int G> __global__ __launch_bounds__(VEC_BLOCK) void logprobs_grad_narrow_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    const int g = threadIdx.x & (G - 1);
    const int64_t rows = VEC_BLOCK / G;
    for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / G; row < a.n; row += (int64_t)gridDim.x * rows) {
        RowGrad<A> w;
        w.load(a, row);
        A sum = A(0);
        for (int t = 0; t < a.m; ++t) sum += given_weight<A>(a, row * a.m + t, a.labels[row * a.m + t]);
        w.G += sum;
        const T *z = (const T *)a.Z + row * a.ldz;
        T *dz = (T *)a.dZ + row * a.lddz;
        const uint32_t *mask = a.allowed ? a.allowed + row * a.ld_allowed : nullptr;
        for (int c = g; c < a.width; c += G) {
            A x = A(0);
            if (!w.empty && (!mask || allowed_bit(mask, c))) {
                x = w.at((A)z[c]);
                for (int t = 0; t < a.m; ++t)
                    if (a.labels[row * a.m + t] == c) x += given_weight<A>(a, row * a.m + t, c);
            }
            dz[c] = (T)x;
        }
    }
}

template <typename F> hipError_t by_type(int dtype, F f)
{
    switch (dtype) {
    case SSN_F32: f(float()); break;
    case SSN_F64: f(double()); break;
    case SSN_F16: f(_Float16()); break;
    default: f(__bf16()); break;
    }
    return hipGetLastError();
}
template <typename F> void by_lanes(int C, int per_lane, F f)
{
    const int need = (C + per_lane - 1) / per_lane;
    if (need <= 1) f(std::integral_constant<int, 1>());
    else if (need <= 2) f(std::integral_constant<int, 2>());
    else if (need <= 4) f(std::integral_constant<int, 4>());
    else if (need <= 8) f(std::integral_constant<int, 8>());
    else if (need <= 16) f(std::integral_constant<int, 16>());
    else if (need <= 32) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
}

constexpr int64_t MAX_GRID = 1 << 20, MAX_ROWS = 65535;        // workgroups of one launch; longer work loops

dim3 row_grid(int64_t per_row, int64_t n) { return dim3((unsigned)per_row, (unsigned)(n < MAX_ROWS ? n : MAX_ROWS)); }

}  // namespace

// Which form serves a call: a pure function of the sizes and the type.
void logprobs_plan(int dtype, int64_t n, int64_t C, int64_t width, int k, int num_cus, LogprobsArgs *a)
{
    const int es = dtype == SSN_F64 ? 8 : dtype == SSN_F32 ? 4 : 2;
    const int64_t step = WAVE * (16 / es);
    a->parts = 1;
    a->waves = 0;
    a->per_wave = 0;
    if (C <= WAVE * NARROW_PER_LANE) return;
    const int64_t steps = (width + step - 1) / step;                   // loads of a whole wave that the row takes
    const int most = dtype == SSN_F64 ? 8 : 16, ahead = dtype == SSN_F64 ? 2 : 4;
    // Figures in us on 256 compute units.  Rows enough to fill the chip: as few waves per row as keep its loads in flight, since
    // joining them costs (bf16, one / four / eight waves: 3000 rows of 4096 9.4 / 11.9 / 17.7, of 12288 17.7 / 19.3 / 22.0;
    // 600 of 12288 10.8 / 7.3 / 7.5; 3000 of 32768 42.9 / 41.5 / 41.8, of 65536 77.5 / 76.7 / 72.6; sixteen 103).  Rows of
    // eight loads or less are one wave's however few (100 of 2048 4.1 / 4.1, of 4096 5.1 / 4.3, less than the call costs the host).
    // Fewer rows than compute units: all the waves a workgroup may have (100 of 8192 bf16: eight 4.5, sixteen 5.2; of 65536
    // 9.1, 8.7), and several workgroups per row where each wave still has loads for one round of AHEAD (one row of 131072
    // fp32, five alternatives: one workgroup 19.4, eight 10.7; of 40960 10.8, four 10.4; of 32000 9.4, two 10.3, since the
    // join is a launch of its own).
    if (steps <= 8 || (steps <= 24 && n >= 8 * num_cus)) {
        a->waves = 1;
    } else if (n >= 2 * num_cus) {
        a->waves = steps <= 64 ? 4 : 8;
    } else if (n >= num_cus) {
        a->waves = 8;
    } else {
        a->waves = most;
        if (steps > 2 * most * ahead) {
            int64_t parts = (steps + most * ahead - 1) / (most * ahead);
            if (parts > num_cus / n) parts = num_cus / n;
            if (parts > LOGPROBS_MAX_PARTS) parts = LOGPROBS_MAX_PARTS;
            a->parts = (int)parts;
        }
    }
    const int64_t shares = (int64_t)a->parts * a->waves;
    a->per_wave = (steps + shares - 1) / shares * step;
}

int64_t logprobs_workspace(int dtype, int64_t n, int k, const LogprobsArgs &a)
{
    if (a.parts <= 1) return 0;
    const int64_t es = dtype == SSN_F64 ? 8 : 4;
    return n * a.parts * (3 * es + (int64_t)k * (es + 4));
}

hipError_t launch_logprobs(int dtype, LogprobsArgs &a, void *workspace, hipStream_t st)
{
    const int64_t items = a.n * a.parts;
    if (a.parts > 1) {
        const int64_t es = dtype == SSN_F64 ? 8 : 4;
        a.ws_stat = workspace;
        a.ws_val = (char *)workspace + items * 3 * es;
        a.ws_id = (int32_t *)((char *)a.ws_val + items * a.k * es);
    }
    const dim3 grid = row_grid(a.parts, a.n);
    return by_type(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        if (!a.waves) {
            by_lanes((int)a.C, NARROW_PER_LANE, [&](auto lanes) {
                constexpr int G = decltype(lanes)::value;
                const int64_t rows = VEC_BLOCK / G, b = (a.n + rows - 1) / rows;
                hipLaunchKernelGGL((logprobs_narrow_kernel<T, G>), dim3((unsigned)(b < MAX_GRID ? b : MAX_GRID)), dim3(VEC_BLOCK),
                                   0, st, a);
            });
            return;
        }
        auto wide = [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            if (a.k) hipLaunchKernelGGL((logprobs_wide_kernel<T, W, true>), grid, dim3(W * WAVE), 0, st, a);
            else hipLaunchKernelGGL((logprobs_wide_kernel<T, W, false>), grid, dim3(W * WAVE), 0, st, a);
        };
        if (a.waves == 1) wide(std::integral_constant<int, 1>());
        else if (a.waves == 4) wide(std::integral_constant<int, 4>());
        else if (a.waves == 8) wide(std::integral_constant<int, 8>());
        else if constexpr (sizeof(T) < 8) wide(std::integral_constant<int, 16>());
        if (a.parts > 1) {
            const dim3 rows((unsigned)(a.n < MAX_GRID ? a.n : MAX_GRID));
            if (a.k) hipLaunchKernelGGL((logprobs_join_kernel<T, true>), rows, dim3(VEC_BLOCK), 0, st, a);
            else hipLaunchKernelGGL((logprobs_join_kernel<T, false>), rows, dim3(WAVE), 0, st, a);
        }
    });
}

hipError_t launch_logprobs_grad(int dtype, const LogprobsArgs &a, hipStream_t st)
{
    return by_type(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        if (a.width <= WAVE * 4) {
            by_lanes((int)a.width, 4, [&](auto lanes) {
                constexpr int G = decltype(lanes)::value;
                const int64_t rows = VEC_BLOCK / G, b = (a.n + rows - 1) / rows;
                hipLaunchKernelGGL((logprobs_grad_narrow_kernel<T, G>), dim3((unsigned)(b < MAX_GRID ? b : MAX_GRID)),
                                   dim3(VEC_BLOCK), 0, st, a);
            });
            return;
        }
        // A short row is one wave's (bf16, one wave / four: 20000 rows of 2048 27 / 49 us, 1000 of 3000 5.6 / 5.5 us).  A
        // workgroup takes two rounds of loads, the second of which is on its way while the first is worked on (8192 x 65536
        // bf16: one round 470 us, two 357 us, four 400 us), or one where two would leave compute units without work
        // (4 x 32000: 3.4 and 4.4 us).  Rows of up to 256 classes share waves (20000 fp32 rows of 100: 9.9 us, a wave each
        // 12.9 us; of 256 17.2 and 12.6 us).
        LogprobsArgs b = a;
        auto go = [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            const int64_t round = W * WAVE * Vec<T>::E * GRAD_AHEAD;
            b.per_wave = a.n * ((a.width + 2 * round - 1) / (2 * round)) >= 1024 ? 2 * round : round;
            hipLaunchKernelGGL((logprobs_grad_wide_kernel<T, W>), row_grid((a.width + b.per_wave - 1) / b.per_wave, a.n), dim3(W * WAVE),
                               0, st, b);
        };
        if (a.width * (int64_t)sizeof(T) <= 4096) go(std::integral_constant<int, 1>());
        else go(std::integral_constant<int, 4>());
    });
}

}  // namespace ssn
