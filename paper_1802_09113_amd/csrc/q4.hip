// Margins Z = X W with the p-by-K weight block W held in 4 bits: a sign and one of eight magnitudes {0, 1/2, 1, 3/2, 2, 3, 4, 6}
// per weight, and one bfloat16 scale per group of 32, 64 or 128 features of a class.
//
// Why these magnitudes: gfx950 converts two such codes to bfloat16 or half precision in one instruction, exactly, and
// both types feed the matrix cores.  A product of a code's number with a bfloat16 / half value is exact in fp32, so a
// group's sum over its features is an fp32 sum of exact products; the scale is applied to that sum in fp32.  Rows in
// fp32 are split into three bfloat16 parts of eight significant bits each, x = x0 + x1 + x2 exactly, and take three
// products.
//
// Layout: tiles of 16 classes, blocks of 128 features; a block of a tile is 1 KB, 16 bytes for each lane (g, o) =
// (lane / 16, lane % 16): word j of them holds features 128 b + 32 j + 8 g + 0..7 of class 16 t + o, which is lane (g, o)'s
// share of the right operand of one 16x16x32 matrix instruction.  A wave reads the block with one load of 16 bytes per
// lane; one, two or four matrix instructions in a row lie inside a group.
#include "ssn_internal.h"

#include <type_traits>

namespace ssn {

namespace {

constexpr int WAVE = 64, TILE = 16, BLOCK = 128;

typedef uint32_t Raw __attribute__((ext_vector_type(4)));
typedef Raw RawAt2 __attribute__((aligned(2)));
typedef Raw RawAt4 __attribute__((aligned(4)));
typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H2 __attribute__((ext_vector_type(2)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// the rows' side: eight consecutive features of one row as one or three matrix operands
template <typename T> struct Rows;
template <> struct Rows<__bf16> {
    static constexpr int PIECES = 1;
    typedef B8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w)
    {
        const B2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
        const B2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
        return Op{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ void load(const __bf16 *x, Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, (Raw) * (const RawAt2 *)x); }
    static __device__ __forceinline__ F4 mul(Op x, Op w, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};
template <> struct Rows<_Float16> {
    static constexpr int PIECES = 1;
    typedef H8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w)
    {
        const H2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
        const H2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
        return Op{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ void load(const _Float16 *x, Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, (Raw) * (const RawAt2 *)x); }
    static __device__ __forceinline__ F4 mul(Op x, Op w, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0); }
};
template <> struct Rows<float> {
    static constexpr int PIECES = 3;
    typedef B8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w) { return Rows<__bf16>::codes(w); }
    static __device__ __forceinline__ void load(const float *x, Op (&o)[3])
    {
        const Raw r[2] = {*(const RawAt4 *)x, *(const RawAt4 *)(x + 4)};
        uint32_t part[3][4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            uint32_t top[2][3];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t u = r[(e + i) / 4][(e + i) % 4];
                const float v = __uint_as_float(u), v0 = __uint_as_float(u & 0xffff0000u);
                // cut, not rounded: x0 never overflows, and what is left has eight significant bits fewer.  +-inf - (+-inf)
                // is no part of the value: 0 there
                const float v1 = __builtin_isinf(v) ? 0.0f : v - v0;
                const float w1 = __uint_as_float(__float_as_uint(v1) & 0xffff0000u);
                top[i][0] = u, top[i][1] = __float_as_uint(v1), top[i][2] = __float_as_uint(v1 - w1);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) part[k][e / 2] = (top[0][k] >> 16) | (top[1][k] & 0xffff0000u);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) o[k] = __builtin_bit_cast(Op, Raw{part[k][0], part[k][1], part[k][2], part[k][3]});
    }
    static __device__ __forceinline__ F4 mul(Op x, Op w, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};

template <typename T> __device__ __forceinline__ T zero_of() { return (T)0.0f; }

// features k .. k + 7 of a row of p; zeros behind the end
template <typename T> __device__ __forceinline__ void row_operand(const T *x, int64_t k, int64_t p, typename Rows<T>::Op (&o)[Rows<T>::PIECES])
{
    if (k + 8 <= p) {
        Rows<T>::load(x + k, o);
    } else {
        T tail[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) tail[e] = k + e < p ? x[k + e] : zero_of<T>();
        Rows<T>::load(tail, o);
    }
}

__device__ __forceinline__ void store_margin(void *Z, int zdtype, int64_t at, float v)
{
    // one rounding, to nearest, of the finished fp32 sum
    if (zdtype == SSN_F32) ((float *)Z)[at] = v;
    else if (zdtype == SSN_F16) ((_Float16 *)Z)[at] = (_Float16)v;
    else ((__bf16 *)Z)[at] = (__bf16)v;
}

// Four waves share a stretch of the blocks of OT tiles and add their sums in a fixed order.  Row r of a group of 16 stands
// at place 4 (r % 4) + r / 4 of the matrix operand: its sums are then in register r / 4 of lane group r % 4, and up to
// four rows need one register of the four (USED = 1).
constexpr int Q4_WAVES = 4;
template <typename T, int GROUP, int RT, int USED, int OT>
__global__ __launch_bounds__(Q4_WAVES *WAVE) void q4_stream_kernel(Q4Args a)
{
    typedef typename Rows<T>::Op Op;
    constexpr int PIECES = Rows<T>::PIECES, PER = GROUP / 32, GROUPS = BLOCK / GROUP;
    __shared__ float sums[Q4_WAVES][RT * 4 * USED][OT * TILE];
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, o = lane & 15, g = lane >> 4;
    const int64_t blocks = (a.p + BLOCK - 1) / BLOCK, tiles = (a.K + TILE - 1) / TILE;
    const int64_t t0 = (int64_t)blockIdx.x * OT, r0 = (int64_t)blockIdx.z * (16 * RT);
    const int64_t shares = (int64_t)a.parts * Q4_WAVES, mine = (int64_t)blockIdx.y * Q4_WAVES + wave;
    const int64_t first = blocks * mine / shares, last = blocks * (mine + 1) / shares;

    const T *x[RT];
    bool live[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int64_t r = r0 + rt * 16 + (o & 3) * 4 + (o >> 2);
        live[rt] = r < a.n;
        x[rt] = (const T *)a.X + (live[rt] ? r : 0) * a.ldx + 8 * g;
    }
    const uint8_t *w[OT];
    const uint16_t *sc[OT];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
        const int64_t t = t0 + ot < tiles ? t0 + ot : tiles - 1;       // a tile twice at the end; its second sums are not stored
        w[ot] = a.packed + t * blocks * (WAVE * 16) + lane * 16;
        sc[ot] = a.scales + t * blocks * (TILE * GROUPS) + o * GROUPS;
    }
    float acc[OT][RT][USED];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < USED; ++i) acc[ot][rt][i] = 0.0f;

#pragma unroll 2
    for (int64_t b = first; b < last; ++b) {
        Raw q[OT];
        uint16_t s[OT][GROUPS];
#pragma unroll
        for (int ot = 0; ot < OT; ++ot) {
            q[ot] = *(const Raw *)(w[ot] + b * (WAVE * 16));
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) s[ot][i] = sc[ot][b * (TILE * GROUPS) + i];
        }
        F4 d[OT][RT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Op xo[RT][PIECES];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                for (int k = 0; k < PIECES; ++k) xo[rt][k] = __builtin_bit_cast(Op, Raw{0, 0, 0, 0});
                if (live[rt]) row_operand<T>(x[rt], b * BLOCK + 32 * j, a.p - 8 * g, xo[rt]);
            }
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) {
                const Op wo = Rows<T>::codes(q[ot][j]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if (j % PER == 0) d[ot][rt] = F4{0, 0, 0, 0};
#pragma unroll
                    for (int k = PIECES - 1; k >= 0; --k) d[ot][rt] = Rows<T>::mul(xo[rt][k], wo, d[ot][rt]);
                    if (j % PER == PER - 1) {
                        const float f = bf16_value(s[ot][j / PER]);
#pragma unroll
                        for (int i = 0; i < USED; ++i) acc[ot][rt][i] = fmaf(f, d[ot][rt][i], acc[ot][rt][i]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int ot = 0; ot < OT; ++ot)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < USED; ++i) sums[wave][rt * 4 * USED + i * 4 + g][ot * TILE + o] = acc[ot][rt][i];
    __syncthreads();
    for (int e = threadIdx.x; e < RT * 4 * USED * OT * TILE; e += Q4_WAVES * WAVE) {
        const int rr = e / (OT * TILE), cc = e % (OT * TILE);
        const int64_t r = r0 + rr, c = t0 * TILE + cc;
        if (r >= a.n || c >= a.K) continue;
        float v = sums[0][rr][cc];
#pragma unroll
        for (int i = 1; i < Q4_WAVES; ++i) v += sums[i][rr][cc];
        if (a.parts > 1) a.ws[((int64_t)blockIdx.y * a.n + r) * a.K + c] = v;
        else store_margin(a.Z, a.zdtype, r * a.ldz + c, v);
    }
}

// the parts' sums in order
__global__ __launch_bounds__(VEC_BLOCK) void q4_join_kernel(Q4Args a)
{
    for (int64_t r = blockIdx.y; r < a.n; r += gridDim.y)
        for (int64_t c = (int64_t)blockIdx.x * VEC_BLOCK + threadIdx.x; c < a.K; c += (int64_t)gridDim.x * VEC_BLOCK) {
            float v = 0.0f;
            for (int i = 0; i < a.parts; ++i) v += a.ws[((int64_t)i * a.n + r) * a.K + c];
            store_margin(a.Z, a.zdtype, r * a.ldz + c, v);
        }
}

// ---- laying a block out in 4 bits --------------------------------------------------------------------------------------
// A scale is the smallest bfloat16 s with 6 s >= the largest magnitude of its group, so no weight is clipped; a code is the
// magnitude nearest to |w| / s, a tie going to the even index.  s times a border between two magnitudes has at most eleven
// significant bits: the comparisons are exact and no quotient is formed for a weight.
constexpr int QUANT_TILES = 2;
template <typename T> struct QuantAcc { typedef float type; };
template <> struct QuantAcc<double> { typedef double type; };

template <typename T>
__global__ __launch_bounds__(VEC_BLOCK) void q4_quantize_kernel(const T *W, int64_t sj, int64_t sc, int64_t p, int64_t K, int group,
                                                                uint8_t *packed, uint16_t *scales)
{
    typedef typename QuantAcc<T>::type A;
    constexpr int CLASSES = QUANT_TILES * TILE;
    __shared__ A w[CLASSES][BLOCK + 1];
    __shared__ float scale[CLASSES][4];
    const int64_t blocks = (p + BLOCK - 1) / BLOCK, tiles = (K + TILE - 1) / TILE;
    const int64_t c0 = (int64_t)blockIdx.x * CLASSES;
    const int groups = BLOCK / group;
    // six times the largest bfloat16, or the largest float: NaN and infinities compare false
    const A reach = sizeof(A) == 8 ? (A)(6.0 * 3.3895313892515355e38) : (A)3.4028234663852886e38f;
    for (int64_t b = blockIdx.y; b < blocks; b += gridDim.y) {
        // neighbouring threads along the shorter stride
        for (int e = threadIdx.x; e < CLASSES * BLOCK; e += VEC_BLOCK) {
            const int c = sj <= sc ? e / BLOCK : e % CLASSES, j = sj <= sc ? e % BLOCK : e / CLASSES;
            const int64_t cc = c0 + c, jj = b * BLOCK + j;
            w[c][j] = cc < K && jj < p ? (A)W[jj * sj + cc * sc] : A(0);
        }
        __syncthreads();
        if (threadIdx.x < CLASSES * groups) {
            const int c = threadIdx.x / groups, i = threadIdx.x % groups;
            A most = A(0);
            bool finite = true;
            for (int j = 0; j < group; ++j) {
                const A v = fabs(w[c][i * group + j]);
                finite = finite && v <= reach;
                most = v > most ? v : most;
            }
            float s = __uint_as_float(__float_as_uint((float)(most / A(6))) & 0xffff0000u);
            if (A(6) * (A)s < most) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
            if (!finite) s = __uint_as_float(0x7fc00000u);
            scale[c][i] = s;
            const int64_t t = c0 / TILE + c / TILE;
            if (t < tiles) scales[((t * blocks + b) * TILE + c % TILE) * groups + i] = (uint16_t)(__float_as_uint(s) >> 16);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < CLASSES * 16; e += VEC_BLOCK) {
            // word j of lane (g, o): 32 consecutive words are the lanes' of one class after the other
            const int j = e & 3, o = (e >> 2) & 15, g = (e >> 6) & 3, tt = e >> 8;
            const int c = tt * TILE + o, k0 = 32 * j + 8 * g;
            const A s = (A)scale[c][k0 / group];
            uint32_t word = 0;
            for (int i = 0; i < 8; ++i) {
                const A v = w[c][k0 + i], m = fabs(v);
                uint32_t code = 0;
                if (s > A(0))
                    code = (m > A(0.25) * s) + (m >= A(0.75) * s) + (m > A(1.25) * s) + (m >= A(1.75) * s) + (m > A(2.5) * s) +
                           (m >= A(3.5) * s) + (m > A(5) * s);
                if (code && v < A(0)) code |= 8u;
                word |= code << (4 * i);
            }
            const int64_t t = c0 / TILE + tt;
            if (t < tiles) ((uint32_t *)packed)[((t * blocks + b) * WAVE + g * 16 + o) * 4 + j] = word;
        }
        __syncthreads();
    }
}

}  // namespace

void q4_plan(int num_cus, Q4Args *a)
{
    const int64_t blocks = (a->p + BLOCK - 1) / BLOCK, tiles = (a->K + TILE - 1) / TILE;
    const int64_t groups = tiles * ((a->n + 63) / 64);
    int64_t parts = 1;
    if (groups < num_cus) parts = (num_cus + groups - 1) / groups;
    const int64_t most = blocks / (Q4_WAVES * 4);                      // four blocks at least for each wave
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    a->parts = (int)(parts < 1 ? 1 : parts);
}

int64_t q4_workspace(const Q4Args &a) { return a.parts > 1 ? (int64_t)a.parts * a.n * a.K * 4 : 0; }

template <typename T, int GROUP> static void q4_launch(const Q4Args &a, hipStream_t st)
{
    const int64_t tiles = (a.K + TILE - 1) / TILE;
    auto go = [&](auto rt, auto used, auto ot) {
        constexpr int RT = decltype(rt)::value, USED = decltype(used)::value, OT = decltype(ot)::value;
        const dim3 grid((unsigned)((tiles + OT - 1) / OT), (unsigned)a.parts, (unsigned)((a.n + 16 * RT - 1) / (16 * RT)));
        hipLaunchKernelGGL((q4_stream_kernel<T, GROUP, RT, USED, OT>), grid, dim3(Q4_WAVES * WAVE), 0, st, a);
    };
    std::integral_constant<int, 1> one;
    std::integral_constant<int, 2> two;
    std::integral_constant<int, 4> four;
    if (a.n <= 4) go(one, one, one);
    else if (a.n <= 16) go(one, four, one);
    else if (a.n <= 32) go(two, four, one);
    else go(four, four, two);
}

hipError_t launch_q4_margins(Q4Args &a, void *workspace, hipStream_t st)
{
    a.ws = (float *)workspace;
    auto by_group = [&](auto tag) {
        typedef decltype(tag) T;
        if (a.group == 32) q4_launch<T, 32>(a, st);
        else if (a.group == 64) q4_launch<T, 64>(a, st);
        else q4_launch<T, 128>(a, st);
    };
    if (a.dtype == SSN_F32) by_group(float());
    else if (a.dtype == SSN_F16) by_group(_Float16());
    else by_group(__bf16());
    if (a.parts > 1) {
        const int64_t bx = (a.K + VEC_BLOCK - 1) / VEC_BLOCK;
        hipLaunchKernelGGL(q4_join_kernel, dim3((unsigned)(bx < 65535 ? bx : 65535), (unsigned)(a.n < 65535 ? a.n : 65535)),
                           dim3(VEC_BLOCK), 0, st, a);
    }
    return hipGetLastError();
}

hipError_t launch_q4_quantize(int dtype, int64_t p, int64_t K, const void *W, int64_t sj, int64_t sc, int group, uint8_t *packed,
                              uint16_t *scales, hipStream_t st)
{
    const int64_t blocks = (p + BLOCK - 1) / BLOCK, ct = (K + QUANT_TILES * TILE - 1) / (QUANT_TILES * TILE);
    const dim3 grid((unsigned)ct, (unsigned)(blocks < 65535 ? blocks : 65535));
    auto go = [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL(q4_quantize_kernel<T>, grid, dim3(VEC_BLOCK), 0, st, (const T *)W, sj, sc, p, K, group, packed, scales);
    };
    if (dtype == SSN_F32) go(float());
    else if (dtype == SSN_F64) go(double());
    else if (dtype == SSN_F16) go(_Float16());
    else go(__bf16());
    return hipGetLastError();
}

}  // namespace ssn
