// Rows of float matrices as 8-bit integers with a scale each, and the sums of a gradient's rows.
//
//   a = max |x_k|,  scale = a * (1/127),  q_k = rint(x_k * (127 * (1/a))),  each operation rounded to float32.
//
// Largest values are found on the bit patterns of |x| as unsigned numbers: the order is that of the values, and an infinity or a NaN comes
// out on top, where a floating-point maximum would lose the NaN.  One float32 division per row, then a product and a rounding per value;
// the rounding is an addition of 1.5 * 2^23, whose low byte then is the code in two's complement.
#include "st_dense.hpp"

namespace st {

static constexpr unsigned ABS_BITS = 0x7fffffffu, INF_BITS = 0x7f800000u;
static constexpr unsigned SMALLEST_TOP = 0x04000000u;     // 2^-119: 127 / a is finite from 2^-121 on

__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & ABS_BITS; }

// multiplier and scale of a row whose largest |value| has the bits `top`
__device__ __forceinline__ float row_multiplier(unsigned top, float* scale)
{
    if (top < SMALLEST_TOP) { *scale = 0.f; return 0.f; }
    if (top >= INF_BITS) { *scale = __uint_as_float(0x7fc00000u); return 0.f; }
    const float a = __uint_as_float(top);
    *scale = a * (1.f / 127.f);
    return 127.f * (1.f / a);
}
// the code in the low byte; a multiplier of 0 stands for a row of zeros or of no numbers, whose codes are 0 whatever v is
__device__ __forceinline__ unsigned code_of(float v, float r) { return r == 0.f ? 0u : __float_as_uint(v * r + 12582912.f); }
__device__ __forceinline__ unsigned pack4(unsigned a, unsigned b, unsigned c, unsigned d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

template <class T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<bf16>(const bf16* p) { return (float)*p; }

// Eight consecutive values from p, of which `n` exist; the others are 0.
template <class T, bool WIDE> __device__ __forceinline__ void load8(const T* p, int64_t n, float (&v)[8])
{
    if (WIDE && n >= 8) {
        if (sizeof(T) == 2) {
            const uint4 u = *(const uint4*)p;
            const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        } else {
            const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? load1(p + i) : 0.f;
}

__device__ __forceinline__ float sum8(const float (&v)[8]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

struct Mask { const void* p; int bf16_; int64_t pitch; };
__device__ __forceinline__ bool mask_on(const Mask& m, int64_t at)
{
    return (m.bf16_ ? (float)((const bf16*)m.p)[at] : ((const float*)m.p)[at]) > 0.f;
}

// --------------------------------------------------------------------------------- rows that lie row by row
// LANES threads a row.  A thread holds four runs of eight values of its row in registers between the search for the largest and the
// rounding, so a row of up to 32 * LANES values is read once; longer rows read the rest twice.
template <class T, bool WIDE, int LANES>
__global__ __launch_bounds__(256) void k_quantize_rows(const T* __restrict__ x, int64_t rows, int64_t len, int64_t pitch, Mask mask,
                                                       int8_t* __restrict__ q, int64_t q_pitch, float* __restrict__ scale,
                                                       float* __restrict__ sum)
{
    constexpr int KEEP = 4;
    __shared__ unsigned tops[4];
    __shared__ double sums[4];
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const bool there = row < rows;
    const T* xr = x + (there ? row : 0) * pitch;
    float v[KEEP][8];
    unsigned top = 0;
    double total = 0.0;
    auto read = [&](int64_t at, float (&w)[8]) {
        load8<T, WIDE>(xr + at, there ? len - at : 0, w);
        if (mask.p)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (there && at + i < len && !mask_on(mask, row * mask.pitch + at + i)) w[i] = 0.f;
    };
#pragma unroll
    for (int j = 0; j < KEEP; ++j) {
        read((int64_t)(j * LANES + lane) * 8, v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[j][i]));
        if (sum) total += sum8(v[j]);
    }
    for (int64_t at = (int64_t)(KEEP * LANES + lane) * 8; at < len; at += LANES * 8) {
        float w[8];
        read(at, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(w[i]));
        if (sum) total += sum8(w);
    }
    if (sum) {
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) total += __shfl_xor(total, d);
        if (LANES == 256) {
            if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
            __syncthreads();
            total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        }
        if (there && lane == 0) sum[row] = (float)total;
    }
    if (!q) return;
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) top = max(top, (unsigned)__shfl_xor((int)top, d));
    if (LANES == 256) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    if (!there) return;
    float s;
    const float r = row_multiplier(top, &s);
    if (lane == 0) scale[row] = s;
    int64_t end = (len + OPERAND_QUANTUM - 1) / OPERAND_QUANTUM * OPERAND_QUANTUM;
    if (end > q_pitch) end = q_pitch;
    int8_t* qr = q + row * q_pitch;
    auto put = [&](int64_t at, const float (&w)[8]) {
        if (at >= end) return;      // (pitch and quantum are multiples of 8: a run is written whole or not at all)
        *(uint2*)(qr + at) = make_uint2(pack4(code_of(w[0], r), code_of(w[1], r), code_of(w[2], r), code_of(w[3], r)),
                                        pack4(code_of(w[4], r), code_of(w[5], r), code_of(w[6], r), code_of(w[7], r)));
    };
#pragma unroll
    for (int j = 0; j < KEEP; ++j) put((int64_t)(j * LANES + lane) * 8, v[j]);
    for (int64_t at = (int64_t)(KEEP * LANES + lane) * 8; at < end; at += LANES * 8) {
        float w[8];
        read(at, w);
        put(at, w);
    }
}

template <class T, bool WIDE>
static void rows_launch(Ctx& c, const QuantSource& s, const Quantized& to, float* sum)
{
    const Mask mask{s.mask, s.mask_bf16, s.mask_pitch};
#define ST_ROWS(L)                                                                                                              \
    ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, WIDE, L>), dim3((unsigned)ceil_div(s.rows, 256 / (L))), dim3(256), 0,     \
              (const T*)s.x, s.rows, s.len, s.pitch, mask, to.q, to.pitch, to.scale, sum)
    if (s.len <= 1024) ST_ROWS(32);
    else if (s.len <= 2048) ST_ROWS(64);
    else ST_ROWS(256);
#undef ST_ROWS
}

static bool wide_ok(const void* p, int64_t pitch, int bf16_, int run)     // runs of `run` values can be loaded at once
{
    const int64_t e = bf16_ ? 2 : 4, bytes = run * e < 16 ? run * e : 16;
    return (uintptr_t)p % bytes == 0 && pitch * e % bytes == 0;
}

void quantize_rows(Ctx& c, const QuantSource& s, const Quantized& to, float* sum)
{
    if (s.rows == 0) return;
    const bool wide = wide_ok(s.x, s.pitch, s.bf16, 8);
    if (s.bf16) { if (wide) rows_launch<bf16, true>(c, s, to, sum); else rows_launch<bf16, false>(c, s, to, sum); }
    else        { if (wide) rows_launch<float, true>(c, s, to, sum); else rows_launch<float, false>(c, s, to, sum); }
}

// ------------------------------------------------------------------------------ rows that lie column by column
// The source is a matrix [len][pitch] whose columns are the operand's rows.  First pass: every block takes 128 columns and one part of
// the contraction and leaves the largest value and the sum of each column's part.  Second pass: tiles of 64 columns x 128 positions go
// through LDS as codes.
int transpose_parts(int64_t rows, int64_t len)
{
    const int64_t across = ceil_div(rows, 128), most = ceil_div(len, 32);
    int64_t parts = ceil_div(1024, across);
    if (parts > 64) parts = 64;
    return (int)(parts > most ? most : parts < 1 ? 1 : parts);
}

template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_column_tops(const T* __restrict__ x, int64_t rows, int64_t len, int64_t pitch, Mask mask,
                                                     int64_t per_part, float* __restrict__ part_max, float* __restrict__ part_sum)
{
    __shared__ unsigned tops[4][128];
    __shared__ float sums[4][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 128 + lane * 2;
    const int64_t from = (int64_t)blockIdx.y * per_part, to = from + per_part < len ? from + per_part : len;
    unsigned t0 = 0, t1 = 0;
    double d0 = 0.0, d1 = 0.0;
    for (int64_t piece = from + wave; piece < to; piece += 256) {     // float32 sums of 64 values, which are added in float64
    float s0 = 0.f, s1 = 0.f;
    for (int64_t k = piece; k < to && k < piece + 256; k += 4) {
        float a = 0.f, b = 0.f;
        if (WIDE && col + 1 < rows) {
            if (sizeof(T) == 2) {
                const unsigned u = *(const unsigned*)(x + k * pitch + col);
                a = __uint_as_float(u << 16); b = __uint_as_float(u & 0xffff0000u);
            } else {
                const float2 u = *(const float2*)(x + k * pitch + col);
                a = u.x; b = u.y;
            }
        } else {
            if (col < rows) a = load1(x + k * pitch + col);
            if (col + 1 < rows) b = load1(x + k * pitch + col + 1);
        }
        if (mask.p) {
            if (col < rows && !mask_on(mask, k * mask.pitch + col)) a = 0.f;
            if (col + 1 < rows && !mask_on(mask, k * mask.pitch + col + 1)) b = 0.f;
        }
        t0 = max(t0, abs_bits(a)); t1 = max(t1, abs_bits(b));
        s0 += a; s1 += b;
    }
    d0 += s0; d1 += s1;
    }
    tops[wave][lane * 2] = t0; tops[wave][lane * 2 + 1] = t1;
    sums[wave][lane * 2] = (float)d0; sums[wave][lane * 2 + 1] = (float)d1;
    __syncthreads();
    const int64_t mine = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (threadIdx.x < 128 && mine < rows) {
        const int i = threadIdx.x;
        if (part_max) part_max[(int64_t)blockIdx.y * rows + mine] = __uint_as_float(max(max(tops[0][i], tops[1][i]), max(tops[2][i], tops[3][i])));
        if (part_sum) part_sum[(int64_t)blockIdx.y * rows + mine] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    }
}

template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_quantize_transposed(const T* __restrict__ x, int64_t rows, int64_t len, int64_t pitch, Mask mask,
                                                             int parts, unsigned len_tiles, const float* __restrict__ part_max,
                                                             const float* __restrict__ part_sum, int8_t* __restrict__ q, int64_t q_pitch,
                                                             float* __restrict__ scale, float* __restrict__ sum)
{
    __shared__ unsigned tops[4][64];
    __shared__ float mult[64];
    __shared__ unsigned tile[64][33];       // codes of 4 positions a word; 33: columns of the tile on different banks
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned row_tile = blockIdx.x / len_tiles, len_tile = blockIdx.x - row_tile * len_tiles;
    const int64_t row0 = (int64_t)row_tile * 64, k0 = (int64_t)len_tile * 128;
    const int64_t mine = row0 + lane;
    unsigned top = 0;
    if (mine < rows)
        for (int p = wave; p < parts; p += 4) top = max(top, __float_as_uint(part_max[(int64_t)p * rows + mine]));
    tops[wave][lane] = top;
    __syncthreads();
    if (wave == 0) {
        float s;
        mult[lane] = row_multiplier(max(max(tops[0][lane], tops[1][lane]), max(tops[2][lane], tops[3][lane])), &s);
        if (len_tile == 0 && mine < rows) scale[mine] = s;
    }
    if (wave == 1 && len_tile == 0 && sum && mine < rows) {
        double t = 0.0;
        for (int p = 0; p < parts; ++p) t += part_sum[(int64_t)p * rows + mine];
        sum[mine] = (float)t;
    }
    __syncthreads();
    const float r = mult[lane];
#pragma unroll 4
    for (int g = wave; g < 32; g += 4) {    // four positions of the contraction, one column a lane
        unsigned c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = k0 + g * 4 + i;
            float v = 0.f;
            if (k < len && mine < rows) {
                v = load1(x + k * pitch + mine);
                if (mask.p && !mask_on(mask, k * mask.pitch + mine)) v = 0.f;
            }
            c[i] = code_of(v, r);
        }
        tile[lane][g] = pack4(c[0], c[1], c[2], c[3]);
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {           // a row's 128 bytes by eight lanes
        const int t = threadIdx.x + h * 256, rr = t >> 3, w = (t & 7) * 4;
        const int64_t row = row0 + rr, at = k0 + w * 4;
        if (row < rows && at < q_pitch)
            *(uint4*)(q + row * q_pitch + at) = make_uint4(tile[rr][w], tile[rr][w + 1], tile[rr][w + 2], tile[rr][w + 3]);
    }
}

__global__ __launch_bounds__(256) void k_join_sums(int64_t rows, int parts, const float* __restrict__ part_sum, float* __restrict__ sum)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows) return;
    double t = 0.0;
    for (int p = 0; p < parts; ++p) t += part_sum[(int64_t)p * rows + i];
    sum[i] = (float)t;
}

template <class T, bool WIDE>
static void tops_launch(Ctx& c, const QuantSource& s, float* part_max, float* part_sum)
{
    const Mask mask{s.mask, s.mask_bf16, s.mask_pitch};
    const int parts = transpose_parts(s.rows, s.len);
    ST_LAUNCH(c, "column_tops", (k_column_tops<T, WIDE>), dim3((unsigned)ceil_div(s.rows, 128), parts), dim3(256), 0, (const T*)s.x, s.rows,
              s.len, s.pitch, mask, ceil_div(s.len, parts), part_max, part_sum);
}
template <class T, bool WIDE>
static void transposed_launch(Ctx& c, const QuantSource& s, const Quantized& to, float* part_max, float* part_sum, float* sum)
{
    const Mask mask{s.mask, s.mask_bf16, s.mask_pitch};
    ST_LAUNCH(c, "quantize_transposed", (k_quantize_transposed<T, WIDE>), dim3((unsigned)(ceil_div(s.rows, 64) * ceil_div(s.len, 128))),
              dim3(256), 0, (const T*)s.x, s.rows, s.len, s.pitch, mask, transpose_parts(s.rows, s.len), (unsigned)ceil_div(s.len, 128),
              part_max, part_sum, to.q, to.pitch, to.scale, sum);
}
static void tops(Ctx& c, const QuantSource& s, float* part_max, float* part_sum)
{
    const bool wide = wide_ok(s.x, s.pitch, s.bf16, 2);
    if (s.bf16) { if (wide) tops_launch<bf16, true>(c, s, part_max, part_sum); else tops_launch<bf16, false>(c, s, part_max, part_sum); }
    else        { if (wide) tops_launch<float, true>(c, s, part_max, part_sum); else tops_launch<float, false>(c, s, part_max, part_sum); }
}

void quantize_transposed(Ctx& c, const QuantSource& s, const Quantized& to, float* part_max, float* part_sum, float* sum)
{
    tops(c, s, part_max, sum ? part_sum : nullptr);
    if (s.bf16) transposed_launch<bf16, false>(c, s, to, part_max, part_sum, sum);
    else        transposed_launch<float, false>(c, s, to, part_max, part_sum, sum);
}

void column_sums(Ctx& c, const QuantSource& s, float* part_sum, float* sum)
{
    tops(c, s, nullptr, part_sum);
    ST_LAUNCH(c, "join_sums", k_join_sums, dim3((unsigned)ceil_div(s.rows, 256)), dim3(256), 0, s.rows, transpose_parts(s.rows, s.len), part_sum, sum);
}

__global__ __launch_bounds__(256) void k_fill_zero(float* __restrict__ p, int64_t rows, int64_t cols, int64_t pitch)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * pitch + i % cols] = 0.f;
}
void fill_zero(Ctx& c, float* p, int64_t rows, int64_t cols, int64_t pitch)
{
    const int64_t blocks = ceil_div(rows * cols, 2048);
    ST_LAUNCH(c, "fill_zero", k_fill_zero, dim3((unsigned)(blocks > 4096 ? 4096 : blocks)), dim3(256), 0, p, rows, cols, pitch);
}

}  // namespace st
