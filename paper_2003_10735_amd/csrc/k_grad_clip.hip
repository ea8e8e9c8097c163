// The 2-norm of many gradients, and the gradients clipped by it.  A launch takes up to CLIP_PER_LAUNCH tensors, whose pointers travel with its
// arguments.  The norm has to be known before the first value can be written, so the list is read twice: 436 M bfloat16 values 146 + 290 us, 6.0
// TB/s each, which is what bounds it; 77.6 M values in odd tensors into float32 29 + 72 us (5.3 and 6.4 TB/s).  One head, 445 075 values in six
// tensors, 9.3 us a call: two launches, the second behind the first's sums.
#include "st_clip.hpp"
#include "st_lists.hpp"
#include "st_quantize.hpp"

#include <math.h>
#include <algorithm>

namespace st {

constexpr int CLIP_PER_LAUNCH = 120, CLIP_BLOCKS = 2048, CLIP_READS = 1 << 14;
struct ClipList {
    const void* g[CLIP_PER_LAUNCH]; void* out[CLIP_PER_LAUNCH]; long long n[CLIP_PER_LAUNCH];
    unsigned first[CLIP_PER_LAUNCH + 1];       // first tile of each
    uint8_t types[CLIP_PER_LAUNCH];            // bit 0: gradients in bfloat16, bit 1: results
    int count;
};
static_assert(sizeof(ClipList) + 128 <= 4096, "kernel arguments");
// values of a tile: small lists are spread over more blocks
static int clip_tile(int64_t all) { return all <= (int64_t)CLIP_BLOCKS * 2048 ? 2048 : 8192; }

// Squares and their sums in float64: no square of a finite gradient is infinite or vanishes, and the order of the sums does not show.
template <class G, int RUNS> __device__ __forceinline__ double tile_squares(const void* p, long long n, long long base)
{
    Raw8<G> v[RUNS];
    load_row((const G*)p, n, [&](int j) { return base + j * 2048; }, v);
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < RUNS; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) { const double d = (double)v[j][k]; s = __builtin_fma(d, d, s); }
    return s;
}
__device__ __forceinline__ double sum_of_parts(const double* __restrict__ parts, int n, double* sums)
{
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) s += parts[i];
    return block_sum(s, sums);
}
template <int RUNS> __global__ __launch_bounds__(256) void k_clip_squares(const ClipList l, unsigned tiles, double* __restrict__ parts)
{
    __shared__ double sums[4];
    // a block's tiles follow one another, so that the tensor is searched once
    const unsigned each = tiles / gridDim.x, rest = tiles - each * gridDim.x;
    unsigned tile = blockIdx.x * each + min(blockIdx.x, rest);
    const unsigned end = tile + each + (blockIdx.x < rest ? 1 : 0);
    int i = tensor_of<CLIP_PER_LAUNCH>(l.first, l.count, tile);
    double s = 0.0;
    for (; tile < end; ++tile) {
        while (i + 1 < l.count && tile >= l.first[i + 1]) ++i;
        const long long base = (long long)(tile - l.first[i]) * (RUNS * 2048) + threadIdx.x * 8;
        s += l.types[i] & 1 ? tile_squares<bf16, RUNS>(l.g[i], l.n[i], base) : tile_squares<float, RUNS>(l.g[i], l.n[i], base);
    }
    s = block_sum(s, sums);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// All parts as one, behind the last.  Every block of every launch reads all parts otherwise, which grows with the square of the list; one block that adds
// them is a launch of 10 - 20 us.  Without it and with it, us a call: 240 tensors of 200 000 values (2 launches, 4096 parts) 85 and 106, 800 of 20 000
// (7, 2400) 71 and 70 - 84, 480 of 200 000 (4, 8192) 191 - 234 and 172 - 216, 2000 of 2000 (17, 2000) 161 - 164 and 120, 10 000 of 1000 (84, 10 000) 920 and 710, 65 536 of
// 1000 (547, 65 536) 9220 and 4760 - 5300.  So it runs where launches times parts pass CLIP_READS.
__global__ __launch_bounds__(256) void k_clip_norm(double* __restrict__ parts, int n)
{
    __shared__ double sums[4];
    const double s = sum_of_parts(parts, n, sums);
    if (threadIdx.x == 0) parts[n] = s;
}

// The norm from its parts, by every block in the same order, and the factor on the gradients.
struct ClipFactor { double norm, factor; };
__device__ __forceinline__ ClipFactor clip_factor(const ClipRule& r, const double* __restrict__ parts, int n, double* sums)
{
    const double norm = sqrt(sum_of_parts(parts, n, sums)) * r.scale;
    return {norm, r.max_norm > 0 && norm > r.max_norm && norm < __builtin_inf() ? r.scale * (r.max_norm / norm) : r.scale};
}

// A thread's values of a tile on their way: asked for, and later scaled and stored.  Runs are as long as 16 bytes of the wider of the two
// types, so that a wavefront's stores are whole lines: eight values where both are bfloat16, else four.  (436 M bfloat16 values into float32 with runs
// of eight 299 us, most of it in halves of lines.)
template <int RUNS> struct Pending { Run<bf16, 8> b8[RUNS]; Run<bf16, 4> b4[2 * RUNS]; Run<float, 4> f4[2 * RUNS]; };
constexpr int BOTH_BF16 = 3;
template <int V> __device__ __forceinline__ long long run_at(long long tile_base, int j) { return tile_base + j * (256 * V) + threadIdx.x * V; }
template <int V, class G, int COUNT> __device__ __forceinline__ void ask_runs(const void* g, long long n, long long base, Run<G, V> (&v)[COUNT])
{
    if (n < V) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) { const long long at = run_at<V>(base, j); v[j].load_short((const G*)g + at, at < n ? (int)(n - at) : 0); }
        return;
    }
#pragma unroll
    for (int j = 0; j < COUNT; ++j) v[j].template load<true>((const G*)g + run_start<V, long long>(run_at<V>(base, j), n));
}
template <int RUNS> __device__ __forceinline__ void ask_tile(const ClipList& l, unsigned tile, int i, Pending<RUNS>& p)
{
    const long long base = (long long)(tile - l.first[i]) * (RUNS * 2048);
    if (l.types[i] == BOTH_BF16) ask_runs<8>(l.g[i], l.n[i], base, p.b8);
    else if (l.types[i] & 1) ask_runs<4>(l.g[i], l.n[i], base, p.b4);
    else ask_runs<4>(l.g[i], l.n[i], base, p.f4);
}
template <class O, int V, class G, int COUNT> __device__ __forceinline__ void store_runs(void* q, long long n, long long base, Run<G, V> (&v)[COUNT], float c1, float c2)
{
    O* o = (O*)q;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
        const long long at = run_at<V>(base, j);
        if (at >= n) continue;
        if (at + V > n && n >= V) v[j].down((int)(at - (n - V)));
        float u[V];
#pragma unroll
        for (int k = 0; k < V; ++k) u[k] = v[j][k] * c1 * c2;
        if (at + V <= n) {
            typedef O OV __attribute__((ext_vector_type(V)));
            typedef OV OVany __attribute__((aligned(sizeof(O))));
            OV w;
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = from_f32<O>(u[k]);
            __builtin_nontemporal_store(w, (OVany*)(o + at));
        } else
#pragma unroll
            for (int k = 0; k < V; ++k) if (at + k < n) o[at + k] = from_f32<O>(u[k]);
    }
}
template <int RUNS> __device__ __forceinline__ void store_tile(const ClipList& l, unsigned tile, int i, Pending<RUNS>& p, float c1, float c2)
{
    const long long n = l.n[i], base = (long long)(tile - l.first[i]) * (RUNS * 2048);
    switch (l.types[i]) {
    case 0: store_runs<float, 4>(l.out[i], n, base, p.f4, c1, c2); break;
    case 1: store_runs<float, 4>(l.out[i], n, base, p.b4, c1, c2); break;
    case 2: store_runs<bf16, 4>(l.out[i], n, base, p.f4, c1, c2); break;
    default: store_runs<bf16, 8>(l.out[i], n, base, p.b8, c1, c2); break;
    }
}
// The blocks go through the list side by side; a block's first tile is on its way while it adds the norm's parts.
template <int RUNS> __global__ __launch_bounds__(256) void k_clip_scale(const ClipList l, const ClipRule r, unsigned tiles, const double* __restrict__ parts, int n_parts)
{
    __shared__ double sums[4];
    Pending<RUNS> p;
    unsigned tile = blockIdx.x;
    int i = tile < tiles ? __builtin_amdgcn_readfirstlane(tensor_of<CLIP_PER_LAUNCH>(l.first, l.count, tile)) : 0;
    if (tile < tiles) ask_tile(l, tile, i, p);
    const ClipFactor c = clip_factor(r, parts, n_parts, sums);
    if (r.norm && blockIdx.x == 0 && threadIdx.x == 0) *r.norm = (float)c.norm;
    // (a factor that float32 does not hold is applied in two steps)
    const float factor = (float)c.factor;
    const bool plain = fabsf(factor) >= 0x1p-120f;
    const float c1 = plain ? factor : (float)(c.factor * 0x1p100), c2 = plain ? 1.f : 0x1p-100f;
    while (tile < tiles) {
        if (c.factor != 1.0 || l.g[i] != l.out[i]) store_tile(l, tile, i, p, c1, c2);
        tile += gridDim.x;
        if (tile >= tiles) break;
        while (i + 1 < l.count && tile >= l.first[i + 1]) ++i;
        ask_tile(l, tile, i, p);
    }
}

// The lists of the launches that the tensors from *next on need: those without values are left out.
static ClipList next_list(const st_grad_tensor* t, int n, int* next, int64_t tile, unsigned* tiles)
{
    ClipList l{};
    unsigned at = 0;
    for (; *next < n && l.count < CLIP_PER_LAUNCH; ++*next) {
        const st_grad_tensor& x = t[*next];
        if (x.n == 0) continue;
        const int i = l.count++;
        l.g[i] = x.grad; l.out[i] = x.out; l.n[i] = x.n; l.first[i] = at;
        l.types[i] = (x.grad_dtype == ST_BF16 ? 1 : 0) | (x.out_dtype == ST_BF16 ? 2 : 0);
        at += (unsigned)ceil_div(x.n, tile);
    }
    l.first[l.count] = at;
    *tiles = at;
    return l;
}
static int64_t all_values(const st_grad_tensor* t, int n)
{
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += t[i].n;
    return all;
}
int64_t clip_parts(const st_grad_tensor* t, int n)
{
    const int64_t tile = clip_tile(all_values(t, n));
    int64_t parts = 0;
    for (int next = 0; next < n;) {
        int64_t at = 0;
        for (int count = 0; next < n && count < CLIP_PER_LAUNCH; ++next) if (t[next].n) { at += ceil_div(t[next].n, tile); ++count; }
        parts += std::min<int64_t>(at, CLIP_BLOCKS);
    }
    return parts;
}
void grad_clip(Ctx& c, const st_grad_tensor* t, int n, const ClipRule& r, double* parts)
{
    const int64_t tile = clip_tile(all_values(t, n));
    int64_t n_parts = 0, launches = 0;
    unsigned tiles = 0;
    for (int next = 0; next < n;) {
        const ClipList l = next_list(t, n, &next, tile, &tiles);
        if (!tiles) continue;
        ++launches;
        const unsigned blocks = std::min<unsigned>(tiles, CLIP_BLOCKS);
        if (tile == 2048) ST_LAUNCH(c, "clip_squares", k_clip_squares<1>, dim3(blocks), dim3(256), 0, l, tiles, parts + n_parts);
        else ST_LAUNCH(c, "clip_squares", k_clip_squares<4>, dim3(blocks), dim3(256), 0, l, tiles, parts + n_parts);
        n_parts += blocks;
    }
    if (r.write && launches * n_parts > CLIP_READS) {
        ST_LAUNCH(c, "clip_norm", k_clip_norm, dim3(1), dim3(256), 0, parts, (int)n_parts);
        parts += n_parts;
        n_parts = 1;
    }
    ClipRule rule = r;
    for (int next = r.write ? 0 : n; next < n || rule.norm;) {      // the first launch writes the norm, if only that
        const ClipList l = next_list(t, n, &next, tile, &tiles);
        const unsigned blocks = std::min<unsigned>(std::max(tiles, 1u), CLIP_BLOCKS);
        if (tiles || rule.norm) {
            if (tile == 2048) ST_LAUNCH(c, "clip_scale", k_clip_scale<1>, dim3(blocks), dim3(256), 0, l, rule, tiles, parts, (int)n_parts);
            else ST_LAUNCH(c, "clip_scale", k_clip_scale<4>, dim3(blocks), dim3(256), 0, l, rule, tiles, parts, (int)n_parts);
        }
        rule.norm = nullptr;
    }
}

}  // namespace st
