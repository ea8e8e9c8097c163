// Rows of float matrices as 8-bit integers with a scale each, and the sums of a gradient's rows.
//
//   a = max |x_k|,  scale = a * (1/127),  q_k = rint(x_k * (127 * (1/a))),  each operation rounded to float32.
//
// Largest values are found on the bit patterns of |x| as unsigned numbers: the order is that of the values, and an infinity or a NaN comes
// out on top, where a floating-point maximum would lose the NaN.  One float32 division per row, then a product and a rounding per value;
// the rounding is an addition of 1.5 * 2^23, whose low byte then is the code in two's complement.
//
// A call's sources go through two launches at most.  The first quantises the sources whose rows lie along memory, each row read once; of
// a source that is to be transposed it finds the largest value (and the sum) of each row's parts.  The second transposes those through
// LDS as codes.  (Sources that share a launch do not wait for one another: a backward pass has four, of which some are a few tiles.)
#include "st_quantize.hpp"

#include <type_traits>

namespace st {

struct Job {
    const void *x, *mask;
    int64_t pitch, mask_pitch, rows, len, q_pitch, per_part;
    int8_t* q;
    float *scale, *sum, *part_max, *part_sum;
    int parts;
    unsigned len_tiles;
    uint8_t bf16_, mask_bf16, along;
};
struct Jobs { unsigned first1[4], first2[4]; int n; Job job[4]; };      // first block of each job in the two launches

// Four neighbouring values, one load.
template <class T> struct Raw4;
template <> struct Raw4<bf16> {
    u32x2 u;
    __device__ __forceinline__ void load(const bf16* p) { u = *(const u32x2_2*)p; }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16); }
};
template <> struct Raw4<float> {
    f32x4_t u;
    __device__ __forceinline__ void load(const float* p) { u = *(const f32x4_4*)p; }
    __device__ __forceinline__ float operator[](int i) const { return u[i]; }
};
template <> struct Raw4<void> {};      // no mask

// Four values at `at` of position `line`, of which `n` exist, zero where the mask is not positive.
template <class T> __device__ __forceinline__ void read(const Job& j, int64_t line, int64_t at, int64_t n, float (&v)[4])
{
    const int count = n < 4 ? (int)n : 4;
    load4((const T*)j.x + line * j.pitch + at, count, v);
    if (!j.mask) return;
    float m[4];
    if (j.mask_bf16) load4((const bf16*)j.mask + line * j.mask_pitch + at, count, m);
    else load4((const float*)j.mask + line * j.mask_pitch + at, count, m);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = m[i] > 0.f ? v[i] : 0.f;
}
// COUNT fours, `step` positions apart, all under way before the first is used.  M: the mask's type, or void.
template <class T, class M, int COUNT>
__device__ __forceinline__ void read_all(const Job& j, int64_t line, int step, int64_t at, float (&v)[COUNT][4])
{
    Raw4<T> x[COUNT];
    Raw4<M> m[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        x[i].load((const T*)j.x + (line + i * step) * j.pitch + at);
        if constexpr (!std::is_void<M>::value) m[i].load((const M*)j.mask + (line + i * step) * j.mask_pitch + at);
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[i][e] = x[i][e];
            if constexpr (!std::is_void<M>::value) v[i][e] = m[i][e] > 0.f ? v[i][e] : 0.f;
        }
}
template <class M, class T> __device__ __forceinline__ void clear_masked(const M* m, int n, Raw8<T>& v)
{
    Raw8<M> on;
    on.load(m, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) if (!(on[i] > 0.f)) v.clear(i);
}
template <class T> __device__ __forceinline__ float sum8(const Raw8<T>& v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

struct Shared {
    union {
        struct { unsigned tops[4]; double sums[4]; } rows;
        struct { unsigned tops[16][64]; float sums[16][64]; } parts;
        struct { unsigned tops[4][64]; double sums[4][64]; float mult[64]; unsigned tile[64][33]; } turn;   // 33: rows begin on other banks
    };
};

// ------------------------------------------------------------------------------------ rows that lie along memory
// LANES threads a row.  A thread holds KEEP runs of eight values of its row, as they came, between the search for the largest and the
// rounding, so a row of up to 8 * KEEP * LANES values is read once; longer rows read the rest twice.  A wavefront takes a row of up to 4096
// bfloat16 values by itself: no barrier, eight loads under way.
template <class T, int LANES, int KEEP> __device__ __forceinline__ void rows_role(const Job& j, unsigned block, Shared& sh)
{
    constexpr int MORE = 4;      // runs under way beyond those
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)block * (256 / LANES) + threadIdx.x / LANES;
    const bool there = row < j.rows;
    const int len = (int)j.len;
    const T* x = (const T*)j.x + row * j.pitch;
    unsigned top = 0;
    double total = 0.0;
    auto load = [&](int at, Raw8<T>& v) { v.load(x + at, there ? len - at : 0); };
    auto mask = [&](int at, Raw8<T>& v) {
        if (!j.mask) return;
        const int n = there ? len - at : 0;
        if (j.mask_bf16) clear_masked((const bf16*)j.mask + row * j.mask_pitch + at, n, v);
        else clear_masked((const float*)j.mask + row * j.mask_pitch + at, n, v);
    };
    auto see = [&](const Raw8<T>& v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
        if (j.sum) total += sum8(v);
    };
    Raw8<T> v[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) load((k * LANES + lane) * 8, v[k]);
#pragma unroll
    for (int k = 0; k < KEEP; ++k) { mask((k * LANES + lane) * 8, v[k]); see(v[k]); }
    for (int at = (KEEP * LANES + lane) * 8; at < len; at += MORE * LANES * 8) {
        Raw8<T> w[MORE];
#pragma unroll
        for (int k = 0; k < MORE; ++k) load(at + k * LANES * 8, w[k]);
#pragma unroll
        for (int k = 0; k < MORE; ++k) { mask(at + k * LANES * 8, w[k]); see(w[k]); }
    }
    if (j.sum) {
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) total += __shfl_xor(total, d);
        if (LANES == 256) {
            if ((threadIdx.x & 63) == 0) sh.rows.sums[threadIdx.x >> 6] = total;
            __syncthreads();
            total = (sh.rows.sums[0] + sh.rows.sums[1]) + (sh.rows.sums[2] + sh.rows.sums[3]);
        }
        if (there && lane == 0) j.sum[row] = (float)total;
    }
    if (!j.q) return;
    top = LANES == 32 ? half_max(top) : wave_max(top);
    if (LANES == 256) {
        if ((threadIdx.x & 63) == 0) sh.rows.tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(sh.rows.tops[0], sh.rows.tops[1]), max(sh.rows.tops[2], sh.rows.tops[3]));
    }
    if (!there) return;
    float s;
    const float r = row_multiplier(top, &s);
    if (lane == 0) j.scale[row] = s;
    const int64_t padded = (j.len + OPERAND_QUANTUM - 1) / OPERAND_QUANTUM * OPERAND_QUANTUM;
    const int end = (int)(padded < j.q_pitch ? padded : j.q_pitch);
    int8_t* qr = j.q + row * j.q_pitch;
    auto put = [&](int at, const Raw8<T>& w) {
        if (at >= end) return;      // (pitch and quantum are multiples of 8: a run is written whole or not at all)
        *(uint2*)(qr + at) = make_uint2(pack4(code_of(w[0], r), code_of(w[1], r), code_of(w[2], r), code_of(w[3], r)),
                                        pack4(code_of(w[4], r), code_of(w[5], r), code_of(w[6], r), code_of(w[7], r)));
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k) v[k].repack();
#pragma unroll
    for (int k = 0; k < KEEP; ++k) put((k * LANES + lane) * 8, v[k]);
    for (int at = (KEEP * LANES + lane) * 8; at < end; at += MORE * LANES * 8) {
        Raw8<T> w[MORE];
#pragma unroll
        for (int k = 0; k < MORE; ++k) load(at + k * LANES * 8, w[k]);
#pragma unroll
        for (int k = 0; k < MORE; ++k) { mask(at + k * LANES * 8, w[k]); put(at + k * LANES * 8, w[k]); }
    }
}
template <class T> constexpr int row_keep() { return sizeof(T) == 2 ? 8 : 4; }
static __host__ __device__ __forceinline__ int row_lanes(int64_t len, int is_bf16) { return len <= 1024 ? 32 : len <= (is_bf16 ? 4096 : 2048) ? 64 : 256; }

// --------------------------------------------------------------------------------------- rows that lie across it
// The source is a matrix [len][pitch] whose columns are the operand's rows.  Sixteen threads take 64 columns of a position, sixteen
// positions at once: whole lines of memory are read.  A block leaves the largest value and the sum of 64 columns over one part.
template <class T, class M> __device__ __forceinline__ void parts_loop(const Job& j, int64_t col, int64_t from, int64_t to, int group, bool whole,
                                                                       unsigned (&top)[4], double (&total)[4])
{
    for (int64_t piece = from + group; piece < to; piece += 1024) {     // float32 sums of 64 values, added in float64
        float s[4] = {};
        const int64_t end = piece + 1024 < to ? piece + 1024 : to;
        int64_t k = piece;
        auto see = [&](const float (&v)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { top[e] = max(top[e], abs_bits(v[e])); s[e] += v[e]; }
        };
        if (whole)
            for (; k + 48 < end; k += 64) {
                float v[4][4];
                read_all<T, M, 4>(j, k, 16, col, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) see(v[i]);
            }
        for (; k < end; k += 16) {
            float v[4];
            read<T>(j, k, col, j.rows - col, v);
            see(v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) total[e] += s[e];
    }
}
template <class T> __device__ __forceinline__ void parts_role(const Job& j, unsigned block, Shared& sh)
{
    const unsigned tile = block / (unsigned)j.parts, part = block - tile * (unsigned)j.parts;
    const int c = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
    const int64_t col = (int64_t)tile * 64 + c;
    const int64_t from = part * j.per_part, to = from + j.per_part < j.len ? from + j.per_part : j.len;
    const bool whole = col + 4 <= j.rows;
    unsigned top[4] = {};
    double total[4] = {};
    if (col < j.rows) {
        if (!j.mask) parts_loop<T, void>(j, col, from, to, group, whole, top, total);
        else if (j.mask_bf16) parts_loop<T, bf16>(j, col, from, to, group, whole, top, total);
        else parts_loop<T, float>(j, col, from, to, group, whole, top, total);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { sh.parts.tops[group][c + i] = top[i]; sh.parts.sums[group][c + i] = (float)total[i]; }
    __syncthreads();
    const int64_t mine = (int64_t)tile * 64 + threadIdx.x;
    if (threadIdx.x < 64 && mine < j.rows) {
        unsigned t = 0;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) { t = max(t, sh.parts.tops[i][threadIdx.x]); s += sh.parts.sums[i][threadIdx.x]; }
        if (j.part_max) j.part_max[(int64_t)part * j.rows + mine] = __uint_as_float(t);
        if (j.part_sum) j.part_sum[(int64_t)part * j.rows + mine] = (float)s;
    }
}

// Tiles of 64 columns x 128 positions.  A thread takes eight positions of four columns: two words of codes for each of four rows.
template <class T> __device__ __forceinline__ void turn_role(const Job& j, unsigned block, Shared& sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned row_tile = block / j.len_tiles, len_tile = block - row_tile * j.len_tiles;
    const int64_t row0 = (int64_t)row_tile * 64, k0 = (int64_t)len_tile * 128;
    const int64_t mine = row0 + lane;
    const bool sums = j.sum && len_tile == 0;
    const int c = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
    float v[8][4] = {};
    if (j.q && row0 + c < j.rows) {
        const int64_t k = k0 + group * 8;
        if (row0 + c + 4 <= j.rows && k + 8 <= j.len) {
            if (!j.mask) read_all<T, void, 8>(j, k, 1, row0 + c, v);
            else if (j.mask_bf16) read_all<T, bf16, 8>(j, k, 1, row0 + c, v);
            else read_all<T, float, 8>(j, k, 1, row0 + c, v);
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < j.len) read<T>(j, k + i, row0 + c, j.rows - row0 - c, v[i]);
    }
    unsigned top = 0;
    double total = 0.0;
    if (mine < j.rows) {
        if (j.q)
#pragma unroll 8
            for (int p = wave; p < j.parts; p += 4) top = max(top, __float_as_uint(j.part_max[(int64_t)p * j.rows + mine]));
        if (sums)
            for (int p = wave; p < j.parts; p += 4) total += j.part_sum[(int64_t)p * j.rows + mine];
    }
    sh.turn.tops[wave][lane] = top;
    sh.turn.sums[wave][lane] = total;
    __syncthreads();
    if (wave == 0) {
        float s;
        sh.turn.mult[lane] = row_multiplier(max(max(sh.turn.tops[0][lane], sh.turn.tops[1][lane]), max(sh.turn.tops[2][lane], sh.turn.tops[3][lane])), &s);
        if (len_tile == 0 && j.q && mine < j.rows) j.scale[mine] = s;
    }
    if (wave == 1 && sums && mine < j.rows)
        j.sum[mine] = (float)((sh.turn.sums[0][lane] + sh.turn.sums[1][lane]) + (sh.turn.sums[2][lane] + sh.turn.sums[3][lane]));
    if (!j.q) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = sh.turn.mult[c + i];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            sh.turn.tile[c + i][group * 2 + h] = pack4(code_of(v[h * 4][i], r), code_of(v[h * 4 + 1][i], r), code_of(v[h * 4 + 2][i], r),
                                                       code_of(v[h * 4 + 3][i], r));
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {           // a row's 128 bytes by eight lanes
        const int t = threadIdx.x + h * 256, rr = t >> 3, w = (t & 7) * 4;
        const int64_t row = row0 + rr, at = k0 + w * 4;
        if (row < j.rows && at < j.q_pitch)
            *(uint4*)(j.q + row * j.q_pitch + at) =
                make_uint4(sh.turn.tile[rr][w], sh.turn.tile[rr][w + 1], sh.turn.tile[rr][w + 2], sh.turn.tile[rr][w + 3]);
    }
}

template <class T> __device__ __forceinline__ void rows_any(const Job& j, unsigned block, Shared& sh)
{
    const int lanes = row_lanes(j.len, sizeof(T) == 2);
    if (lanes == 32) rows_role<T, 32, 4>(j, block, sh);
    else if (lanes == 64) rows_role<T, 64, row_keep<T>()>(j, block, sh);
    else rows_role<T, 256, 4>(j, block, sh);
}
template <class T> __device__ __forceinline__ void first_role(const Job& j, unsigned block, Shared& sh)
{
    if (!j.along) parts_role<T>(j, block, sh);
    else rows_any<T>(j, block, sh);
}
__global__ __launch_bounds__(256) void k_quantize_first(const Jobs jobs)
{
    __shared__ Shared sh;
    int i = 0;
    while (i + 1 < jobs.n && blockIdx.x >= jobs.first1[i + 1]) ++i;
    const Job& j = jobs.job[i];
    if (j.bf16_) first_role<bf16>(j, blockIdx.x - jobs.first1[i], sh); else first_role<float>(j, blockIdx.x - jobs.first1[i], sh);
}
// one source that lies along memory: the forward pass
template <class T, int LANES, int KEEP> __global__ __launch_bounds__(256) void k_quantize_rows(const Job j)
{
    __shared__ Shared sh;
    rows_role<T, LANES, KEEP>(j, blockIdx.x, sh);
}
template <class T> static void rows_launch(Ctx& c, const Job& j, unsigned blocks)
{
    switch (row_lanes(j.len, sizeof(T) == 2)) {
    case 32: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 32, 4>), dim3(blocks), dim3(256), 0, j); break;
    case 64: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 64, row_keep<T>()>), dim3(blocks), dim3(256), 0, j); break;
    default: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 256, 4>), dim3(blocks), dim3(256), 0, j);
    }
}
__global__ __launch_bounds__(256) void k_quantize_turn(const Jobs jobs)
{
    __shared__ Shared sh;
    int i = 0;
    while (i + 1 < jobs.n && blockIdx.x >= jobs.first2[i + 1]) ++i;
    const Job& j = jobs.job[i];
    if (j.bf16_) turn_role<bf16>(j, blockIdx.x - jobs.first2[i], sh); else turn_role<float>(j, blockIdx.x - jobs.first2[i], sh);
}

// ------------------------------------------------------------------------------------------------------------- host
// Blocks enough to fill the card, parts of 64 positions at least; the second launch reads every part's value of each of its rows.
int transpose_parts(int64_t rows, int64_t len)
{
    const int64_t across = ceil_div(rows, 64), most = ceil_div(len, 64);
    int64_t parts = ceil_div(1024, across);
    if (parts > 128) parts = 128;
    return (int)(parts > most ? most : parts < 1 ? 1 : parts);
}

void quantize(Ctx& c, const QuantTask* tasks, int n)
{
    Jobs jobs;
    jobs.n = 0;
    // sources that lie along memory first, so that the second launch has the others in consecutive places
    int64_t blocks1 = 0, blocks2 = 0;
    for (int pass = 1; pass >= 0; --pass)
        for (int i = 0; i < n; ++i) {
            const QuantTask& t = tasks[i];
            const QuantSource& s = t.s;
            if (s.along != pass || s.rows == 0) continue;
            jobs.first1[jobs.n] = (unsigned)blocks1; jobs.first2[jobs.n] = (unsigned)blocks2;
            Job& j = jobs.job[jobs.n++];
            j = Job{s.x, s.mask, s.pitch, s.mask_pitch, s.rows, s.len, t.to.pitch, 0, t.to.q, t.to.scale, t.sum, t.to.q ? t.part_max : nullptr,
                    t.sum ? t.part_sum : nullptr, 1, 1, (uint8_t)s.bf16, (uint8_t)s.mask_bf16, (uint8_t)s.along};
            if (s.along) { blocks1 += ceil_div(s.rows, 256 / row_lanes(s.len, s.bf16)); continue; }
            j.parts = transpose_parts(s.rows, s.len);
            j.per_part = ceil_div(s.len, j.parts);
            j.len_tiles = t.to.q ? (unsigned)ceil_div(s.len, 128) : 1;
            blocks1 += ceil_div(s.rows, 64) * j.parts;
            blocks2 += ceil_div(s.rows, 64) * j.len_tiles;
        }
    if (jobs.n == 1 && jobs.job[0].along) {
        if (jobs.job[0].bf16_) rows_launch<bf16>(c, jobs.job[0], (unsigned)blocks1); else rows_launch<float>(c, jobs.job[0], (unsigned)blocks1);
    } else if (blocks1) ST_LAUNCH(c, "quantize_first", k_quantize_first, dim3((unsigned)blocks1), dim3(256), 0, jobs);
    if (!blocks2) return;
    Jobs turn;
    turn.n = 0;
    for (int i = 0; i < jobs.n; ++i)
        if (!jobs.job[i].along) { turn.first2[turn.n] = jobs.first2[i]; turn.job[turn.n++] = jobs.job[i]; }
    ST_LAUNCH(c, "quantize_turn", k_quantize_turn, dim3((unsigned)blocks2), dim3(256), 0, turn);
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
