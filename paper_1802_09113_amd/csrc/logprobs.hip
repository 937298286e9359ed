// Log probabilities of given classes, entropy and top alternatives of rows of margins, and their gradient.
//
// A row z of C margins (a class that is not allowed counts as -inf, the reference class as 0) has, as in eq. (8), (9),
//   M = max_c z_c,  s = sum_c e^{z_c - M},  t = sum_c e^{z_c - M} (z_c - M) <= 0,
//   log p_y = (z_y - M) - log s,  H = -sum_c p_c log p_c = log s - t / s  (two terms >= 0: nothing cancels),
// and log s in [0, log C] is kept apart from M, so that log p_y carries no rounding of a large log-sum-exp.  One pass over
// the row: every lane keeps (M, s, t) of what it has seen and rescales s and t when its M grows; pairs are joined the same
// way across lanes, waves and workgroups.  s is NaN exactly when a margin is NaN or +inf, and 0 exactly when no class is
// left (the largest margin contributes e^0 = 1).  All of it in fp32 for fp32, fp16 and bf16 margins, in fp64 for fp64.
#include "ssn_internal.h"
#include "ssn_math.h"

#include <type_traits>

namespace ssn {

namespace {

constexpr int WAVE = 64;
constexpr int NARROW_PER_LANE = 8;      // margins per lane of the narrow form

template <typename T> struct Acc { typedef float type; };
template <> struct Acc<double> { typedef double type; };

// 16 bytes of margins at an address aligned to an element only
typedef uint32_t Raw __attribute__((ext_vector_type(4)));
typedef Raw RawAt2 __attribute__((aligned(2)));
typedef Raw RawAt4 __attribute__((aligned(4)));
template <typename T> struct Vec {
    static constexpr int E = 16 / sizeof(T);
    typedef typename std::conditional<sizeof(T) == 2, RawAt2, RawAt4>::type RawAt;
    static __device__ __forceinline__ Raw load(const T *p) { return *(const RawAt *)p; }
    static __device__ __forceinline__ void store(T *p, Raw v) { *(RawAt *)p = v; }
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
template <typename A> __device__ __forceinline__ A sum_over(A x, int lanes)
{
    for (int o = lanes / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, WAVE);
    return x;
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
        s = sum_over(s, WAVE);
        t = sum_over(t, WAVE);
    }
};

// One row's answer.  s == 0: no class is left; s != s: the row holds NaN or +inf at an allowed class.
template <typename A> struct Answer {
    A M, L, s, t;
    __device__ __forceinline__ Answer(const Stat<A> &q) : M(q.M), s(q.s), t(q.t) { L = s == A(0) ? A(0) : log_sum(s); }
    __device__ __forceinline__ A maxpart() const { return s == A(0) ? minus_inf(A()) : s == s ? M : s; }
    __device__ __forceinline__ A logpart() const { return L; }
    __device__ __forceinline__ A entropy() const { return s == A(0) ? A(0) : L - t / s; }
    __device__ __forceinline__ A logp(A z) const
    {
        if (!(s == s)) return s;
        return s == A(0) || z == minus_inf(A()) ? minus_inf(A()) : (z - M) - L;
    }
};

__device__ __forceinline__ bool allowed_bit(const uint32_t *mask, int64_t c) { return (mask[c >> 5] >> (c & 31)) & 1u; }

// ---- top alternatives: lane i < k of the wave holds the i-th best (value, class) seen, -inf where there is none --------
template <typename A> struct Best {
    A v;
    int id;
    A least;                            // the k-th best value: what does not exceed it is not taken
    __device__ __forceinline__ void init() { v = least = minus_inf(A()), id = -1; }
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
    // the k best of `lists` sorted lists (value and class at [list * k + i]) whose classes ascend from list to list
    __device__ __forceinline__ void merge(const A *vals, const int *ids, int lists, int lane, int k)
    {
        init();
        int h = 0;
        A head = lane < lists ? vals[lane * k] : minus_inf(A());
        int hid = lane < lists ? ids[lane * k] : -1;
        for (int i = 0; i < k; ++i) {
            const A m = wave_max(head);
            if (m == minus_inf(A())) break;
            const int who = __ffsll((unsigned long long)__ballot(head == m)) - 1;
            const int c = __builtin_amdgcn_readlane(hid, who);
            if (lane == i) v = m, id = c;
            if (lane == who) {
                ++h;
                head = h < k ? vals[lane * k + h] : minus_inf(A());
                hid = h < k ? ids[lane * k + h] : -1;
            }
        }
    }
};

template <typename T> __device__ __forceinline__ typename Acc<T>::type margin_of(const LogprobsArgs &a, int64_t row, int64_t c)
{
    typedef typename Acc<T>::type A;
    if (a.allowed && !allowed_bit(a.allowed + row * a.ld_allowed, c)) return minus_inf(A());
    if (c >= a.width) return A(0);                                     // the reference class
    return (A)((const T *)a.Z)[row * a.ldz + c];
}

// the outputs of one row by one wave: zy is the margin of given class `lane` (lanes < m)
template <typename T, bool TOP>
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int64_t row, int lane, const Stat<typename Acc<T>::type> &q,
                                          int y, typename Acc<T>::type zy, const Best<typename Acc<T>::type> &best)
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
        const bool none = !(q.s == q.s) || best.v == minus_inf(A());
        a.top_ids[row * a.k + lane] = none ? -1 : best.id;
        ((A *)a.top_logp)[row * a.k + lane] = w.logp(best.v);
    }
}

// ---- rows of many classes: WAVES waves share a row, or one of `parts` stretches of it ---------------------------------
// Each wave walks a stretch of its own, AHEAD loads of 16 bytes per lane in flight.
template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES *WAVE) void logprobs_wide_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    constexpr int E = Vec<T>::E, STEP = WAVE * E, AHEAD = sizeof(T) == 8 ? 2 : 4;
    __shared__ A sh_stat[WAVES][3];
    __shared__ A sh_val[TOP && WAVES > 1 ? WAVES * WAVE : 1];
    __shared__ int sh_id[TOP && WAVES > 1 ? WAVES * WAVE : 1];
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
    const int part = blockIdx.x;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const T *z = (const T *)a.Z + row * a.ldz;
        const uint32_t *mask = a.allowed ? a.allowed + row * a.ld_allowed : nullptr;
        const int64_t first = ((int64_t)part * WAVES + wave) * a.per_wave;
        const int64_t end = first + a.per_wave < a.width ? first + a.per_wave : a.width;
        // given classes: their margins are on the way while the row is read
        int y = -1;
        A zy = A(0);
        if (a.parts == 1 && wave == 0 && lane < a.m) {
            y = a.labels[row * a.m + lane];
            if (y >= 0 && y < a.C) zy = margin_of<T>(a, row, y);
        }
        Stat<A> q;
        q.init();
        Best<A> best;
        best.init();
        for (int64_t c0 = first; c0 < end; c0 += AHEAD * STEP) {
            Raw raw[AHEAD];
            uint32_t bits[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t c = c0 + u * STEP + lane * E;
                raw[u] = Raw{0, 0, 0, 0};
                bits[u] = 0;
                if (c + E <= end) {
                    raw[u] = Vec<T>::load(z + c);
                    bits[u] = (1u << E) - 1;
                } else if (c < end) {                                  // the row's last, partial vector
                    T tail[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) tail[e] = z[c + e < end ? c + e : end - 1];
                    raw[u] = __builtin_bit_cast(Raw, tail);
                    bits[u] = (1u << (int)(end - c)) - 1;
                }
                if (mask && c < end) bits[u] &= mask[c >> 5] >> (c & 31);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (c0 + u * STEP >= end) break;
                A x[E];
                unpack(raw[u], x, T());
                if (mask || c0 + (u + 1) * STEP > end) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = (bits[u] >> e) & 1u ? x[e] : minus_inf(A());
                }
                A top = x[0];
#pragma unroll
                for (int e = 1; e < E; ++e) top = take_max(top, x[e]);
                q.raise(take_max(q.M, top));
#pragma unroll
                for (int e = 0; e < E; ++e) q.add(x[e]);
                if (TOP) best.take(x, (int)(c0 + u * STEP + lane * E), lane, a.k);
            }
        }
        // the reference class, behind all others
        if (a.reference && part == a.parts - 1 && wave == WAVES - 1 && (!mask || allowed_bit(mask, a.width))) {
            if (lane == 0) {
                q.raise(take_max(q.M, A(0)));
                q.add(A(0));
            }
            if (TOP && A(0) > best.least) best.insert(A(0), (int)a.width, lane, a.k);
        }
        q.join_wave();
        if (WAVES > 1) {
            if (lane == 0) sh_stat[wave][0] = q.M, sh_stat[wave][1] = q.s, sh_stat[wave][2] = q.t;
            if (TOP && lane < a.k) sh_val[wave * a.k + lane] = best.v, sh_id[wave * a.k + lane] = best.id;
            __syncthreads();
            if (wave == 0) {
                q.init();
                if (lane < WAVES) q.M = sh_stat[lane][0], q.s = sh_stat[lane][1], q.t = sh_stat[lane][2];
                q.join_wave();
                if (TOP) best.merge(sh_val, sh_id, WAVES, lane, a.k);
            }
        }
        if (wave == 0) {
            if (a.parts == 1) {
                write_row<T, TOP>(a, row, lane, q, y, zy, best);
            } else {
                const int64_t item = row * a.parts + part;
                if (lane == 0) {
                    A *w = (A *)a.ws_stat + item * 3;
                    w[0] = q.M, w[1] = q.s, w[2] = q.t;
                }
                if (TOP && lane < a.k) ((A *)a.ws_val)[item * a.k + lane] = best.v, a.ws_id[item * a.k + lane] = best.id;
            }
        }
        if (WAVES > 1) __syncthreads();
    }
}

// the parts of a row joined, a wave per row
template <typename T, bool TOP> __global__ __launch_bounds__(WAVE) void logprobs_join_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    __shared__ A sh_val[TOP ? LOGPROBS_MAX_PARTS * WAVE : 1];
    __shared__ int sh_id[TOP ? LOGPROBS_MAX_PARTS * WAVE : 1];
    const int lane = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        int y = -1;
        A zy = A(0);
        if (lane < a.m) {
            y = a.labels[row * a.m + lane];
            if (y >= 0 && y < a.C) zy = margin_of<T>(a, row, y);
        }
        Stat<A> q;
        q.init();
        if (lane < a.parts) {
            const A *w = (const A *)a.ws_stat + (row * a.parts + lane) * 3;
            q.M = w[0], q.s = w[1], q.t = w[2];
        }
        Best<A> best;
        best.init();
        if (TOP) {
            const int64_t at = row * a.parts * a.k;
            for (int i = lane; i < a.parts * a.k; i += WAVE) sh_val[i] = ((const A *)a.ws_val)[at + i], sh_id[i] = a.ws_id[at + i];
            __syncthreads();
        }
        q.join_wave();
        if (TOP) best.merge(sh_val, sh_id, a.parts, lane, a.k);
        write_row<T, TOP>(a, row, lane, q, y, zy, best);
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
        Stat<A> q;
        q.init();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = g + r * G;
            x[r] = live && c < a.C ? margin_of<T>(a, row, c) : minus_inf(A());
        }
#pragma unroll
        for (int r = 0; r < R; ++r) q.M = take_max(q.M, x[r]);
        for (int o = G / 2; o > 0; o >>= 1) q.M = take_max(q.M, __shfl_xor(q.M, o, WAVE));
#pragma unroll
        for (int r = 0; r < R; ++r) q.add(x[r]);
        q.s = sum_over(q.s, G);
        q.t = sum_over(q.t, G);
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
        for (int i = 0; i < a.k; ++i) {                                // the largest margin left, the lowest class first
            A v = minus_inf(A());
            int id = -1;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (x[r] > v) v = x[r], id = g + r * G;
            for (int o = G / 2; o > 0; o >>= 1) {
                const A ov = __shfl_xor(v, o, WAVE);
                const int oid = __shfl_xor(id, o, WAVE);
                if (ov > v || (ov == v && (unsigned)oid < (unsigned)id)) v = ov, id = oid;
            }
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
};
// given class y's weight: none for padding and for a class without probability, NaN for an index that is no class
template <typename A> __device__ __forceinline__ A given_weight(const LogprobsArgs &a, int64_t at, int y)
{
    if (y < 0) return A(0);
    if (y >= a.C) return nan_of(A());
    return ((const A *)a.logp)[at] == minus_inf(A()) ? A(0) : ((const A *)a.dlogp)[at];
}

template <typename T> __global__ __launch_bounds__(VEC_BLOCK) void logprobs_grad_wide_kernel(LogprobsArgs a)
{
    typedef typename Acc<T>::type A;
    constexpr int E = Vec<T>::E, U = 2, TILE = VEC_BLOCK * E * U;
    const int lane = threadIdx.x & (WAVE - 1);
    const int64_t c0 = (int64_t)blockIdx.x * TILE;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const T *z = (const T *)a.Z + row * a.ldz;
        T *dz = (T *)a.dZ + row * a.lddz;
        const uint32_t *mask = a.allowed ? a.allowed + row * a.ld_allowed : nullptr;
        Raw raw[U];
        uint32_t bits[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + (u * VEC_BLOCK + threadIdx.x) * E;
            raw[u] = Raw{0, 0, 0, 0};
            bits[u] = (1u << E) - 1;
            if (c + E <= a.width) {
                raw[u] = Vec<T>::load(z + c);
            } else if (c < a.width) {
                T tail[E];
#pragma unroll
                for (int e = 0; e < E; ++e) tail[e] = z[c + e < a.width ? c + e : a.width - 1];
                raw[u] = __builtin_bit_cast(Raw, tail);
            }
            if (mask && c < a.width) bits[u] = mask[c >> 5] >> (c & 31);
        }
        int y = -1;
        A gy = A(0);
        if (lane < a.m) {
            y = a.labels[row * a.m + lane];
            gy = given_weight<A>(a, row * a.m + lane, y);
        }
        RowGrad<A> w;
        w.load(a, row);
        w.G += sum_over(gy, WAVE);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t cw = c0 + (u * VEC_BLOCK + (threadIdx.x - lane)) * E;     // the wave's stretch
            if (cw >= a.width) break;
            const int64_t c = cw + lane * E;
            A x[E];
            unpack(raw[u], x, T());
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = w.empty || !((bits[u] >> e) & 1u) ? A(0) : w.at(x[e]);
            for (unsigned long long b = __ballot(gy != A(0) && y >= cw && y < cw + WAVE * E); b; b &= b - 1) {
                const int from = __ffsll(b) - 1;
                const int64_t yy = __builtin_amdgcn_readlane(y, from);
                const A g = at_lane(gy, from);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] += c + e == yy ? g : A(0);
            }
            if (c + E <= a.width) {
                Vec<T>::store(dz + c, pack(x, T()));
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c + e < a.width) dz[c + e] = (T)x[e];
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
            A x = w.empty || (mask && !allowed_bit(mask, c)) ? A(0) : w.at((A)z[c]);
            for (int t = 0; t < a.m; ++t)
                if (a.labels[row * a.m + t] == c) x += given_weight<A>(a, row * a.m + t, c);
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
    a->waves = steps <= 8 ? 1 : 4;
    if (n < 2 * num_cus && steps > 16) {
        a->waves = 16;
        int64_t parts = (steps + 16 * 8 - 1) / (16 * 8);
        if (n < num_cus) {
            const int64_t fill = (num_cus + n - 1) / n;
            if (parts < fill) parts = fill;
        }
        if (parts > (steps + 31) / 32) parts = (steps + 31) / 32;
        if (parts > LOGPROBS_MAX_PARTS) parts = LOGPROBS_MAX_PARTS;
        a->parts = (int)parts;
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
        else wide(std::integral_constant<int, 16>());
        if (a.parts > 1) {
            const dim3 rows((unsigned)(a.n < MAX_GRID ? a.n : MAX_GRID));
            if (a.k) hipLaunchKernelGGL((logprobs_join_kernel<T, true>), rows, dim3(WAVE), 0, st, a);
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
        constexpr int TILE = VEC_BLOCK * Vec<T>::E * 2;
        hipLaunchKernelGGL((logprobs_grad_wide_kernel<T>), row_grid((a.width + TILE - 1) / TILE, a.n), dim3(VEC_BLOCK), 0, st, a);
    });
}

}  // namespace ssn
