// Margins Z = X W with the p-by-K weight block W held in 4 bits: a sign and one of eight magnitudes {0, 1/2, 1, 3/2, 2, 3, 4, 6}
// per weight, and one bfloat16 scale per group of 32, 64 or 128 features of a class.
//
// Why these magnitudes: gfx950 converts two such codes to bfloat16 or half precision in one instruction, exactly, and
// both types feed the matrix cores.  A product of a code's number with a bfloat16 / half value is exact in fp32, so a
// group's sum over its features is an fp32 sum of exact products; the scale is applied to that sum in fp32.  Rows in
// fp32 are split into three bfloat16 parts of eight significant bits each, x = x0 + x1 + x2, and take three products.
// That is exact down to the last bit that a bfloat16 number has, 2^-133.
//
// A group's sum is formed before its scale, so it may be 768 times the largest feature where the margin is small.  Bfloat16
// codes are therefore converted to 2^-10 of their numbers, which the instruction does for nothing, and a margin's sum carries
// that factor until it is stored: no finite features overflow, and what a sum loses are its bits below 2^-139.
//
// Layout: tiles of 16 classes, blocks of 128 features; a block of a tile is 1 KB, 16 bytes for each lane (g, o) =
// (lane / 16, lane % 16): word j of them holds features 128 b + 32 j + 8 g + 0..7 of class 16 t + o, which is lane (g, o)'s
// share of the right operand of one 16x16x32 matrix instruction.  A wave reads the block with one load of 16 bytes per
// lane; one, two or four matrix instructions in a row lie inside a group.
//
// What bounds it: for few rows the stream of codes and scales (one row, 8192 x 65536, groups of 32: 302 MB in 62 us in a queue of
// passes, 4.9 TB/s, 57 us in a graph).  For many the matrix cores and the vector units, which convert codes and scale sums, in
// turn, with two waves a SIMD (256 f16 rows, 4096 x 32768, groups of 128: 64 to 69 us, 1000 to 1070 TFLOP/s, where a library product
// of plain f16 matrices reaches 1160; matrix cores 49 % busy, vector units 45 %), the more so in groups of 32 (84 to 87 us).
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
    static constexpr float UNIT = 0.0009765625f;                       // what the codes are multiplied with, 2^-10
    typedef B8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w)
    {
        const B2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, UNIT, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, UNIT, 1);
        const B2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, UNIT, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, UNIT, 3);
        return Op{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ void operand(const Raw (&r)[1], Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, r[0]); }
    static __device__ __forceinline__ void load(const __bf16 *x, Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, (Raw) * (const RawAt2 *)x); }
    static __device__ __forceinline__ F4 mul(Op x, Op w, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};
template <> struct Rows<_Float16> {
    static constexpr int PIECES = 1;
    static constexpr float UNIT = 1.0f;                                // 768 times the largest half is no large float
    typedef H8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w)
    {
        const H2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
        const H2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
        return Op{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ void operand(const Raw (&r)[1], Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, r[0]); }
    static __device__ __forceinline__ void load(const _Float16 *x, Op (&o)[1]) { o[0] = __builtin_bit_cast(Op, (Raw) * (const RawAt2 *)x); }
    static __device__ __forceinline__ F4 mul(Op x, Op w, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0); }
};
template <> struct Rows<float> {
    static constexpr int PIECES = 3;
    static constexpr float UNIT = Rows<__bf16>::UNIT;
    typedef B8 Op;
    static __device__ __forceinline__ Op codes(uint32_t w) { return Rows<__bf16>::codes(w); }
    // the three parts of two features, a word of two bfloat16 numbers each
    static __device__ __forceinline__ void split(const uint32_t (&u)[2], uint32_t (&word)[3])
    {
        uint32_t top[2][3];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float v = __uint_as_float(u[i]), v0 = __uint_as_float(u[i] & 0xffff0000u);
            // cut, not rounded: x0 never overflows, and what is left has eight significant bits fewer.  +-inf - (+-inf) is no
            // part of the value: 0 there
            const float v1 = __builtin_isinf(v) ? 0.0f : v - v0;
            const float w1 = __uint_as_float(__float_as_uint(v1) & 0xffff0000u);
            top[i][0] = u[i], top[i][1] = __float_as_uint(v1), top[i][2] = __float_as_uint(v1 - w1);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) word[k] = (top[0][k] >> 16) | (top[1][k] & 0xffff0000u);
    }
    static __device__ __forceinline__ void load(const float *x, Op (&o)[3])
    {
        const Raw r[2] = {*(const RawAt4 *)x, *(const RawAt4 *)(x + 4)};
        operand(r, o);
    }
    static __device__ __forceinline__ void operand(const Raw (&r)[2], Op (&o)[3])
    {
        uint32_t part[3][4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            uint32_t word[3];
            split({r[e / 4][e % 4], r[e / 4][e % 4 + 1]}, word);
#pragma unroll
            for (int k = 0; k < 3; ++k) part[k][e / 2] = word[k];
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

// eight consecutive margins of a row, of which `left` are inside it
template <typename Z> __device__ __forceinline__ void store_margins(Z *z, int64_t left, const float (&v)[8])
{
    if (left >= 8) {
        Z out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = (Z)v[e];
        Raw r[sizeof(Z) / 2];
        __builtin_memcpy(r, out, sizeof(out));
#pragma unroll
        for (int h = 0; h < (int)sizeof(Z) / 2; ++h) ((RawAt2 *)z)[h] = r[h];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) z[e] = (Z)v[e];
    }
}

// the scales of a class in a block, in one load
template <int GROUPS> struct ScaleWord;
template <> struct ScaleWord<1> { typedef uint16_t type; };
template <> struct ScaleWord<2> { typedef uint32_t type; };
template <> struct ScaleWord<4> { typedef uint64_t type; };

// WAVES waves share a stretch of the blocks of OT tiles and add their sums in a fixed order.  Row r of a group of 16 stands
// at place 4 (r % 4) + r / 4 of the matrix operand: its sums are then in register r / 4 of lane group r % 4, and up to
// four rows need one register of the four (USED = 1).  Places without a row hold the last row again; their sums are not
// stored.
template <typename T, int GROUP, int USED, int OT, int WAVES, int DEPTH>
__global__ __launch_bounds__(WAVES *WAVE) void q4_stream_kernel(Q4Args a)
{
    typedef typename Rows<T>::Op Op;
    constexpr int PIECES = Rows<T>::PIECES, PER = GROUP / 32, GROUPS = BLOCK / GROUP;
    typedef typename ScaleWord<GROUPS>::type Scales;
    __shared__ float sums[WAVES][4 * USED][OT * TILE];
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), o = lane & 15, g = lane >> 4;
    const int64_t blocks = (a.p + BLOCK - 1) / BLOCK, tiles = (a.K + TILE - 1) / TILE, whole = a.p / BLOCK;
    const int64_t t0 = (int64_t)blockIdx.x * OT, r0 = (int64_t)blockIdx.z * 16;
    const int64_t shares = (int64_t)a.parts * WAVES, mine = (int64_t)blockIdx.y * WAVES + wave;
    const int64_t first = blocks * mine / shares, last = blocks * (mine + 1) / shares;

    const int64_t own = r0 + (o & 3) * 4 + (o >> 2);                   // the row at this lane's place
    const T *x = (const T *)a.X + (own < a.n ? own : a.n - 1) * a.ldx + 8 * g;
    const Raw *w[OT];
    const Scales *sc[OT];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
        const int64_t t = t0 + ot < tiles ? t0 + ot : tiles - 1;       // a tile twice at the end; its second sums are not stored
        w[ot] = (const Raw *)a.packed + t * blocks * WAVE;
        sc[ot] = (const Scales *)a.scales + t * blocks * TILE;
    }
    float acc[OT][USED];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot)
#pragma unroll
        for (int i = 0; i < USED; ++i) acc[ot][i] = 0.0f;

    // one block: xo(j) fills the rows' operands of word j
    auto block = [&](const Raw (&q)[OT], const Scales (&s)[OT], auto rows) {
        F4 d[OT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Op xo[PIECES];
            rows(j, xo);
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) {
                const Op wo = Rows<T>::codes(q[ot][j]);
                const float f = bf16_value((uint16_t)(s[ot] >> (16 * (j / PER))));
                if (j % PER == 0) d[ot] = F4{0, 0, 0, 0};
#pragma unroll
                for (int k = PIECES - 1; k >= 0; --k) d[ot] = Rows<T>::mul(xo[k], wo, d[ot]);
                if (j % PER == PER - 1) {
#pragma unroll
                    for (int i = 0; i < USED; ++i) acc[ot][i] = fmaf(f, d[ot][i], acc[ot][i]);
                }
            }
        }
    };
    // fp32 rows, sixteen at most: a lane splits its share of each row once and the wave reads the operands from LDS; to split
    // them where they are used would cost a lane four rows' work for one row
    constexpr bool STAGED = PIECES == 3;
    constexpr int ROWS = 4 * USED, LINE = BLOCK * 2 + 16;              // a row's 128 numbers, 16 bytes apart in the banks
    __shared__ __align__(16) unsigned char stage[STAGED ? WAVES * 3 * ROWS * LINE : 16];
    unsigned char *st = stage + (STAGED ? wave * 3 * ROWS * LINE : 0);
    const int64_t stop = last < whole ? last : whole;
    for (int64_t b = first; b < stop; b += DEPTH) {
        Raw q[DEPTH][OT];
        Scales s[DEPTH][OT];
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            const int64_t bb = b + u < stop ? b + u : stop - 1;        // fetched again where there is no such block
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) {
                q[u][ot] = (w[ot] + bb * WAVE)[lane];
                s[u][ot] = (sc[ot] + bb * TILE)[o];
            }
        }
        if constexpr (STAGED) {
            typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(4)));
            Pair v[DEPTH][ROWS];
#pragma unroll
            for (int u = 0; u < DEPTH; ++u)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const int64_t bb = b + u < stop ? b + u : stop - 1;
                    if (r0 + r < a.n) v[u][r] = *(const Pair *)((const float *)a.X + (r0 + r) * a.ldx + bb * BLOCK + 2 * lane);
                }
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                if (b + u >= stop) break;
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    if (r0 + r < a.n) {
                        uint32_t word[3];
                        Rows<float>::split({v[u][r][0], v[u][r][1]}, word);
#pragma unroll
                        for (int k = 0; k < 3; ++k) *(uint32_t *)(st + (k * ROWS + r) * LINE + 4 * lane) = word[k];
                    }
                // the wave's own LDS, which it reads and writes in order
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                const int row = own < a.n && own - r0 < ROWS ? (int)(own - r0) : 0;
                block(q[u], s[u], [&](int j, Op (&xo)[PIECES]) {
#pragma unroll
                    for (int k = 0; k < PIECES; ++k)
                        xo[k] = __builtin_bit_cast(Op, *(const Raw *)(st + (k * ROWS + row) * LINE + 64 * j + 16 * g));
                });
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            continue;
        }
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (b + u >= stop) break;
            block(q[u], s[u], [&](int j, Op (&xo)[PIECES]) {
                Rows<T>::load(x + (b + u) * BLOCK + 32 * j, xo);
            });
        }
    }
    if (last > whole && first < last) {                                // features end inside the last block
        Raw q[OT];
        Scales s[OT];
#pragma unroll
        for (int ot = 0; ot < OT; ++ot) {
            q[ot] = (w[ot] + whole * WAVE)[lane];
            s[ot] = (sc[ot] + whole * TILE)[o];
        }
        block(q, s, [&](int j, Op (&xo)[PIECES]) {
            row_operand<T>(x, whole * BLOCK + 32 * j, a.p - 8 * g, xo);
        });
    }
#pragma unroll
    for (int ot = 0; ot < OT; ++ot)
#pragma unroll
        for (int i = 0; i < USED; ++i) sums[wave][i * 4 + g][ot * TILE + o] = acc[ot][i];
    __syncthreads();
    for (int e = threadIdx.x; e < 4 * USED * OT * TILE; e += WAVES * WAVE) {
        const int rr = e / (OT * TILE), cc = e % (OT * TILE);
        const int64_t r = r0 + rr, c = t0 * TILE + cc;
        if (r >= a.n || c >= a.K) continue;
        float v = sums[0][rr][cc];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += sums[i][rr][cc];
        if (a.parts > 1) a.ws[((int64_t)blockIdx.y * a.n + r) * a.K + c] = v;
        else store_margin(a.Z, a.zdtype, r * a.ldz + c, v * (1.0f / Rows<T>::UNIT));
    }
}

// More rows: a wave takes 16 RT rows and 64 classes, WM x WN waves side by side share the rows' blocks through LDS, and WK
// such groups take a stretch of the features each and add their sums in order.  Two buffers of rows per group; a row's sixteen
// chunks of 16 bytes are exchanged by the row's number in its tile of sixteen, so that the sixteen lanes that read one chunk
// of sixteen rows meet all banks.  fp32 rows are split on their way into LDS.  The weights come straight from memory in their
// operands' order, one block ahead.  Each group's products are summed in registers of their own and scaled from there.
template <typename T, int GROUP, int RT, int WM, int WN, int WK>
__global__ __launch_bounds__(WM *WN *WK *WAVE) void q4_tile_kernel(Q4Args a)
{
    typedef typename Rows<T>::Op Op;
    constexpr int PIECES = Rows<T>::PIECES, PER = GROUP / 32, GROUPS = BLOCK / GROUP, OT = 4;
    constexpr int SIDE = WM * WN * WAVE, ROWS = 16 * RT * WM, LOADS = ROWS * 16 / SIDE, CLASSES = WN * OT * TILE;
    constexpr int BUFFER = PIECES * ROWS * 16;                         // chunks of a buffer
    static_assert(LOADS * SIDE == ROWS * 16 && LOADS >= 1, "whole rounds of the chunks");
    static_assert(WK == 1 || ROWS * CLASSES * 4 <= 2 * WK * BUFFER * 16, "a group's sums fit the buffers");
    typedef typename ScaleWord<GROUPS>::type Scales;
    constexpr int LINE = OT * TILE + 4, OUT = TILE * LINE / 4;         // a tile row of a wave's results on their way out, in chunks
    __shared__ Raw lds[2 * WK * BUFFER > WM * WN * OUT ? 2 * WK * BUFFER : WM * WN * OUT];
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), o = lane & 15, g = lane >> 4;
    const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN, side = threadIdx.x - wk * SIDE;
    const int blocks = (int)((a.p + BLOCK - 1) / BLOCK), tiles = (int)((a.K + TILE - 1) / TILE), whole = (int)(a.p / BLOCK);
    // workgroups that share weights are neighbours
    const unsigned row_groups = (unsigned)((a.n + ROWS - 1) / ROWS);
    const int64_t r0 = (int64_t)(blockIdx.x % row_groups) * ROWS;
    const int t0 = blockIdx.x / row_groups * (WN * OT) + wn * OT;
    const int shares = a.parts * WK, mine = blockIdx.y * WK + wk;
    const int first = (int)((int64_t)blocks * mine / shares), last = (int)((int64_t)blocks * (mine + 1) / shares);
    const int rounds = (blocks + shares - 1) / shares;                 // of the group with most blocks

    const Raw *w[OT];
    const Scales *sc[OT];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
        const int64_t t = t0 + ot < tiles ? t0 + ot : tiles - 1;
        w[ot] = (const Raw *)a.packed + (t * blocks + first) * WAVE;
        sc[ot] = (const Scales *)a.scales + (t * blocks + first) * TILE;
    }
    // the thread's chunks: row (i SIDE + side) / 16, chunk side % 16
    const int chunk = side & 15, row = side >> 4;
    const T *x[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int64_t r = r0 + row + i * (SIDE / 16);
        x[i] = (const T *)a.X + (r < a.n ? r : a.n - 1) * a.ldx + chunk * 8;
    }
    constexpr int WORDS = sizeof(T) / 2;                               // 16-byte loads of a chunk's features
    Raw xr[LOADS][WORDS], q[OT];
    Scales s[OT];
    auto fetch_rows = [&](int b, int i) {
#pragma unroll
        for (int h = 0; h < WORDS; ++h) xr[i][h] = *(const RawAt2 *)(x[i] + (int64_t)b * BLOCK + h * 4);
    };
    auto fetch_weights = [&](int b, int ot) {
        q[ot] = (w[ot] + (int64_t)(b - first) * WAVE)[lane];
        s[ot] = (sc[ot] + (int64_t)(b - first) * TILE)[o];
    };
    // where the thread's chunks go in a buffer, and where the lane's operands are
    int put[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int rr = row + i * (SIDE / 16);
        put[i] = rr * 16 + (chunk ^ (rr & 15));
    }
    float acc[OT][RT][4];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[ot][rt][i] = 0.0f;
    // what is fetched behind the end (the last whole block of rows, the last block of weights) is not used
    const int start = first < blocks ? first : blocks - 1;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) fetch_rows(start < whole ? start : whole - 1, i);
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) fetch_weights(start, ot);
    for (int i0 = 0; i0 < rounds; ++i0) {
        const int b = first + i0;
        Raw *buf = lds + (2 * wk + (i0 & 1)) * BUFFER;
        if (b == whole) {                                              // the features end inside this block
            const int left = (int)(a.p - (int64_t)b * BLOCK) - chunk * 8;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                T tail[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) tail[e] = e < left ? x[i][(int64_t)b * BLOCK + e] : zero_of<T>();
                __builtin_memcpy(xr[i], tail, sizeof(tail));
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            Op op[PIECES];
            Rows<T>::operand(xr[i], op);
#pragma unroll
            for (int k = 0; k < PIECES; ++k) buf[k * ROWS * 16 + put[i]] = __builtin_bit_cast(Raw, op[k]);
        }
        __syncthreads();                                               // the other buffer's readers are behind this too
        if (b >= last) continue;
        const Raw *at = buf + (wm * 16 * RT + o) * 16;
        Op xo[4][RT][PIECES];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int k = 0; k < PIECES; ++k)
                    xo[j][rt][k] = __builtin_bit_cast(Op, at[(k * ROWS + rt * 16) * 16 + ((4 * j + g) ^ o)]);
        const int next = b + 1 < blocks ? b + 1 : blocks - 1, next_rows = b + 1 < whole ? b + 1 : whole - 1;
        // the next block's loads go out between the products: all at once they would hold the wave up for as long as the
        // products take
#pragma unroll
        for (int ot = 0; ot < OT; ++ot) {
            F4 d[RT];
            const Raw words = q[ot];
            const Scales scales = s[ot];
            fetch_weights(next, ot);
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                if (i * OT / LOADS == ot) fetch_rows(next_rows, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Op wo = Rows<T>::codes(words[j]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    if (j % PER == 0) d[rt] = F4{0, 0, 0, 0};
#pragma unroll
                for (int k = PIECES - 1; k >= 0; --k)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) d[rt] = Rows<T>::mul(xo[j][rt][k], wo, d[rt]);
                if (j % PER == PER - 1) {
                    const float f = bf16_value((uint16_t)(scales >> (16 * (j / PER))));
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[ot][rt][i] = fmaf(f, d[rt][i], acc[ot][rt][i]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (WK > 1) {
        // the groups' sums in order: lane-major, so that neither side waits for a bank
        constexpr int LANES = WM * WN * WAVE;
        F4 *sums = (F4 *)lds;
        for (int k = 1; k < WK; ++k) {
            __syncthreads();                                           // the buffers, or the last group's sums, have been read
            if (wk == k) {
#pragma unroll
                for (int ot = 0; ot < OT; ++ot)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        sums[(ot * RT + rt) * LANES + side] = F4{acc[ot][rt][0], acc[ot][rt][1], acc[ot][rt][2], acc[ot][rt][3]};
            }
            __syncthreads();
            if (wk == 0) {
#pragma unroll
                for (int ot = 0; ot < OT; ++ot)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const F4 v = sums[(ot * RT + rt) * LANES + side];
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[ot][rt][i] += v[i];
                    }
            }
        }
    }
    // Results through LDS, sixteen rows of the wave's 64 classes at a time: eight lanes write eight classes each of a row
    __syncthreads();
    if (wk) return;
    float *out = (float *)(lds + (wm * WN + wn) * OUT);
    const int64_t c = (int64_t)t0 * TILE + (lane & 7) * 8;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int ot = 0; ot < OT; ++ot)
#pragma unroll
            for (int i = 0; i < 4; ++i) out[(4 * g + i) * LINE + ot * TILE + o] = acc[ot][rt][i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int rr = h * 8 + (lane >> 3);
            const int64_t r = r0 + wm * 16 * RT + rt * 16 + rr;
            const F4 lo = *(const F4 *)(out + rr * LINE + (lane & 7) * 8), hi = *(const F4 *)(out + rr * LINE + (lane & 7) * 8 + 4);
            const float u = a.parts > 1 ? 1.0f : 1.0f / Rows<T>::UNIT;
            const float v[8] = {lo[0] * u, lo[1] * u, lo[2] * u, lo[3] * u, hi[0] * u, hi[1] * u, hi[2] * u, hi[3] * u};
            if (r >= a.n || c >= a.K) continue;
            if (a.parts > 1) store_margins((float *)a.ws + ((int64_t)blockIdx.y * a.n + r) * a.K + c, a.K - c, v);
            else if (a.zdtype == SSN_F32) store_margins((float *)a.Z + r * a.ldz + c, a.K - c, v);
            else if (a.zdtype == SSN_F16) store_margins((_Float16 *)a.Z + r * a.ldz + c, a.K - c, v);
            else store_margins((__bf16 *)a.Z + r * a.ldz + c, a.K - c, v);
        }
    }
}

// the parts' sums in order; what the codes were multiplied with is taken out of the margin
__global__ __launch_bounds__(VEC_BLOCK) void q4_join_kernel(Q4Args a)
{
    const float u = a.dtype == SSN_F16 ? 1.0f / Rows<_Float16>::UNIT : 1.0f / Rows<__bf16>::UNIT;
    for (int64_t r = blockIdx.y; r < a.n; r += gridDim.y)
        for (int64_t c = (int64_t)blockIdx.x * VEC_BLOCK + threadIdx.x; c < a.K; c += (int64_t)gridDim.x * VEC_BLOCK) {
            float v = 0.0f;
            for (int i = 0; i < a.parts; ++i) v += a.ws[((int64_t)i * a.n + r) * a.K + c];
            store_margin(a.Z, a.zdtype, r * a.ldz + c, v * u);
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

// Which kernel serves a call, by its sizes and types alone.  Figures: 4096 features, groups of 32 (64 for 5 to 8 float rows) on
// 256 compute units, in us, bfloat16 rows unless float is said; a tile is 16 classes.
//   Few rows take one register in four (up to 4 rows), two (8) or all (16).  Few tiles: one or two a workgroup, so that every
//   compute unit has one.  Many: four a workgroup, which read the rows' operands once.  The border lies where the small
//   workgroups begin to take another turn on the chip; splitting float rows is worth sharing sooner.
//     1 row    one tile / four     8192 classes 5.8 / 8.3    20480 10.3 / 10.9   32768 14.7 / 13.6   65536 34.8 / 26.4
//     4 float  one / four          8192  8.5 / 9.6           12288 12.0 / 10.9   14336 14.2 / 11.3   65536 53.5 / 33.6
//     8        two / four          8192  7.6 / 8.8           16384 11.6 / 10.1   20480 14.3 / 12.4 (1024 features: 4.9 / 5.2)
//     5 float  two / four by eight waves / four by four waves
//              8192 8.6 / 10.0 / 14.1    12288 11.4 / 11.2 / 14.8    24576 17.8 / 16.1 / 17.4    65536 42.8 / 34.2 / 32.3
//              (in groups of 32: 45.4 / 45.5 / 39.2)
//     16       two / four          8192  8.5 / 10.4          12288 12.5 / 10.8   24576 17.9 / 16.1
//     16 float two / four / tile kernel  8192 14.2 / 16.5 / 17.6   12288 24.6 / 16.7 / 18.0   16384 25.8 / 17.4 / 19.2   24576 36.3 / 30.2 / 21.3
//   More float rows: 16 rows by 128 classes, by eight waves (four groups of features) while that makes less than two workgroups
//   a compute unit, by four beyond: 32 rows, 16384 classes 22.9 / 28.1, 32768 43.9 / 40.4, 131072 181 / 150.
//   More 16-bit rows: the largest tile that still gives 5/8 of the compute units a workgroup,
//     32 rows   16 x 128 / 32 x 128       16384 classes 18.4 / 18.4   20480 22.0 / 18.7    32768 30.0 / 23.0
//     64        32 x 128 / 64 x 128       16384 21.6 / 29.5           20480 35.4 / 30.1    32768 41.1 / 30.9
//     64        64 x 128 / 64 x 256       32768 30.9 / 40.8           40960 56.5 / 41.7    65536 65.4 / 51.3
//     128       64 x 256 / 128 x 256      32768 46.3 / 74.1           40960 82.5 / 74.9    65536 100 / 86.7
//   So few classes that most compute units would have nothing: parts of the features, each with 64 blocks (few rows) or 32,
//   joined by a launch of its own (20000 features, 1000 classes, 1 row: one part 10.8, two 9.1, four 7.6; 64 rows: one 51, four
//   20.0, eight 17.4; 8192 features, 1 row: one 4.9, two 5.8).
namespace {
enum Q4Form : int {
    Q4_ROWS4, Q4_ROWS4_WIDE, Q4_ROWS8, Q4_ROWS8_SPLIT, Q4_ROWS8_WIDE, Q4_ROWS16, Q4_ROWS16_WIDE,       // stream kernel
    Q4_TILE16, Q4_TILE16_HALF, Q4_TILE32, Q4_TILE64, Q4_TILE64_WIDE, Q4_TILE128         // tile kernel: rows of a workgroup
};
int64_t groups_of(int64_t n, int64_t K, int rows, int classes) { return (n + rows - 1) / rows * ((K + classes - 1) / classes); }
}  // namespace

void q4_plan(int num_cus, Q4Args *a)
{
    const int64_t blocks = (a->p + BLOCK - 1) / BLOCK, tiles = (a->K + TILE - 1) / TILE, n = a->n, K = a->K;
    const bool split = a->dtype == SSN_F32;
    int64_t groups, share = 64;                                        // workgroups, and blocks that keep one busy
    if (n <= 4) {
        a->form = tiles >= (split ? 7 : 10) * num_cus / 2 ? Q4_ROWS4_WIDE : Q4_ROWS4;
        groups = a->form == Q4_ROWS4 ? tiles : tiles / 4;
    } else if (n <= 8) {
        a->form = tiles >= (split ? 6 : 5) * num_cus ? Q4_ROWS8_WIDE : split && tiles > 2 * num_cus ? Q4_ROWS8_SPLIT : Q4_ROWS8;
        groups = a->form == Q4_ROWS8 ? tiles / 2 + 1 : tiles / 4;
    } else if (a->p < BLOCK || (n <= 16 && (!split || tiles <= 4 * num_cus))) {
        a->form = (split ? tiles > 2 * num_cus : tiles >= 3 * num_cus) ? Q4_ROWS16_WIDE : Q4_ROWS16;
        groups = (tiles / 2 + 1) * ((n + 15) / 16);
    } else if (split) {
        a->form = groups_of(n, K, 16, 128) >= 2 * num_cus ? Q4_TILE16_HALF : Q4_TILE16;
        groups = groups_of(n, K, 16, 128);
    } else {
        const int64_t enough = 5 * num_cus / 8;
        a->form = Q4_TILE16;
        if (n > 64 && groups_of(n, K, 128, 256) >= enough) a->form = Q4_TILE128;
        else if (n > 32 && groups_of(n, K, 64, 256) >= enough) a->form = Q4_TILE64_WIDE;
        else if (n > 32 && groups_of(n, K, 64, 128) >= enough) a->form = Q4_TILE64;
        else if (groups_of(n, K, 32, 128) >= enough) a->form = Q4_TILE32;
        groups = groups_of(n, K, 16, 128);
        share = 32;
    }
    int64_t parts = groups < num_cus / 2 ? num_cus / groups : 1;
    if (parts > blocks / share) parts = blocks / share;
    if (parts > 64) parts = 64;
    a->parts = (int)(parts < 1 ? 1 : parts);
}

int64_t q4_workspace(const Q4Args &a) { return a.parts > 1 ? (int64_t)a.parts * a.n * a.K * 4 : 0; }

// Workgroups of one launch: their threads have to fit 32 bits.  More classes take a launch for each stretch of them.
static constexpr int64_t MAX_GRID = 1 << 20;

// f(arguments, tiles) for stretches of at most `most` tiles of classes.  More than one only where the rows are not split.
template <typename F> static void each_stretch(const Q4Args &a, int64_t most, F f)
{
    const int64_t tiles = (a.K + TILE - 1) / TILE, blocks = (a.p + BLOCK - 1) / BLOCK;
    for (int64_t t = 0; t < tiles; t += most) {
        Q4Args b = a;
        b.packed += t * blocks * (WAVE * sizeof(Raw));
        b.scales += t * blocks * (TILE * BLOCK / a.group);
        b.Z = (char *)a.Z + t * TILE * (a.zdtype == SSN_F32 ? 4 : 2);
        b.K = a.K - t * TILE < most * TILE ? a.K - t * TILE : most * TILE;
        f(b, (b.K + TILE - 1) / TILE);
    }
}

template <typename T, int GROUP> static void q4_launch(const Q4Args &a, hipStream_t st)
{
    constexpr bool SPLIT = sizeof(T) == 4;
    auto stream = [&](auto used, auto ot, auto waves, auto depth) {
        constexpr int USED = decltype(used)::value, OT = decltype(ot)::value, WAVES = decltype(waves)::value;
        each_stretch(a, MAX_GRID * OT, [&](const Q4Args &b, int64_t tiles) {
            const dim3 grid((unsigned)((tiles + OT - 1) / OT), (unsigned)a.parts, (unsigned)((a.n + 15) / 16));
            hipLaunchKernelGGL((q4_stream_kernel<T, GROUP, USED, OT, WAVES, decltype(depth)::value>), grid, dim3(WAVES * WAVE), 0, st, b);
        });
    };
    auto tile = [&](auto rt, auto wm, auto wn, auto wk) {
        constexpr int RT = decltype(rt)::value, WM = decltype(wm)::value, WN = decltype(wn)::value, WK = decltype(wk)::value;
        const int64_t row_groups = (a.n + 16 * RT * WM - 1) / (16 * RT * WM);              // at most 2^15
        each_stretch(a, MAX_GRID / row_groups * (4 * WN), [&](const Q4Args &b, int64_t tiles) {
            const dim3 grid((unsigned)(row_groups * ((tiles + 4 * WN - 1) / (4 * WN))), (unsigned)a.parts);
            hipLaunchKernelGGL((q4_tile_kernel<T, GROUP, RT, WM, WN, WK>), grid, dim3(WM * WN * WK * WAVE), 0, st, b);
        });
    };
    std::integral_constant<int, 1> one;
    std::integral_constant<int, 2> two;
    std::integral_constant<int, 4> four;
    std::integral_constant<int, 8> eight;
    std::integral_constant<int, SPLIT ? 8 : 4> wide;
    switch (a.form) {
    case Q4_ROWS4: stream(one, one, eight, two); return;
    case Q4_ROWS4_WIDE: stream(one, four, wide, one); return;
    case Q4_ROWS8: stream(two, two, eight, one); return;
    case Q4_ROWS8_SPLIT:
        if constexpr (SPLIT) stream(two, four, eight, one);
        return;
    case Q4_ROWS8_WIDE: stream(two, four, four, one); return;
    case Q4_ROWS16: stream(four, two, eight, one); return;
    case Q4_ROWS16_WIDE: stream(four, four, eight, one); return;
    case Q4_TILE16: tile(one, one, two, four); return;
    default: break;
    }
    if constexpr (SPLIT) {
        tile(one, one, two, two);                                      // Q4_TILE16_HALF
    } else {
        if (a.form == Q4_TILE32) tile(two, one, two, four);
        else if (a.form == Q4_TILE64) tile(two, two, two, two);
        else if (a.form == Q4_TILE64_WIDE) tile(four, one, four, two);
        else tile(four, two, four, one);
    }
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
    const int64_t blocks = (p + BLOCK - 1) / BLOCK, most = MAX_GRID * QUANT_TILES * TILE;
    auto go = [&](auto tag) {
        typedef decltype(tag) T;
        for (int64_t c = 0; c < K; c += most) {
            const int64_t t = c / TILE, left = K - c < most ? K - c : most;
            const dim3 grid((unsigned)((left + QUANT_TILES * TILE - 1) / (QUANT_TILES * TILE)), (unsigned)(blocks < 65535 ? blocks : 65535));
            hipLaunchKernelGGL(q4_quantize_kernel<T>, grid, dim3(VEC_BLOCK), 0, st, (const T *)W + c * sc, sj, sc, p, left, group,
                               packed + t * blocks * (WAVE * sizeof(Raw)), scales + t * blocks * (TILE * BLOCK / group));
        }
    };
    if (dtype == SSN_F32) go(float());
    else if (dtype == SSN_F64) go(double());
    else if (dtype == SSN_F16) go(_Float16());
    else go(__bf16());
    return hipGetLastError();
}

}  // namespace ssn
