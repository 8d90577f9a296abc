// decode_paged.hip -- the decode step over a paged cache: its split into ranges of
// long windows, and their join.  The attention is in decode_paged_tiles.hip (pages in
// bf16 or e4m3) and decode_paged_f32.hip.
//
// With t = len_in[s], the working set W_t (Sec. 3.5, eq. online_ws) is the
// window's rows max(0, t - k)..t - 1, the partner t - pi and the new row, which is
// turned by its position (rotary.h), written to its page as row t and attended as
// stored.  Rows whose page is not there (given back) are not in W_t.  H / Hk query heads
// share a key head, and every row read serves them all.
#include <algorithm>

#include "paged_step.h"

namespace pi_attn {

namespace {

// Joins the parts of a query head: every wavefront takes each WAVES-th, four at a
// time.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void join_kernel(PagedStepParams p) {
    constexpr int EPL = D / 64, U = 4;
    __shared__ float s_m[WAVES], s_l[WAVES];
    __shared__ float s_o[WAVES][D];
    const DivMod head_of = divmod(blockIdx.x, p.H);
    const int s = (int)head_of.quot, h = (int)head_of.rem;
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t head = blockIdx.x, heads = (int64_t)p.S * p.H;
    const int t = p.len_in[s];
    const bool in_reach = t >= 0 && t < (int64_t)p.pages.page * p.pages.max_pages;
    // (looked at behind the parts, which need not wait for it)
    const int entry = in_reach ? p.pages.table[(int64_t)s * p.pages.max_pages + p.pages.by_page.div(t)] : -1;
    const int n = in_reach ? ranges_of(p, t - window_lo(t, p.k)) : 0;
    float M = -INFINITY, L = 0.0f, o[EPL] = {};
    for (int x = w; x < n; x += WAVES * U) {
        float2 ml[U];
        float po[U][EPL];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = min(x + u * WAVES, n - 1) * heads + head;
            ml[u] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
#pragma unroll
            for (int e = 0; e < EPL; ++e) po[u][e] = p.part_o[at * D + lane + 64 * e];
        }
        float m_new = M;
#pragma unroll
        for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, x + u * WAVES < n ? ml[u].x : -INFINITY);
        const float a = M == m_new ? 1.0f : __builtin_amdgcn_exp2f(M - m_new);
        M = m_new;
        L *= a;
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] *= a;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x + u * WAVES >= n) break;
            const float b = ml[u].x == M ? 1.0f : __builtin_amdgcn_exp2f(ml[u].x - M);
            L += ml[u].y * b;
#pragma unroll
            for (int e = 0; e < EPL; ++e) o[e] += po[u][e] * b;
        }
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) s_o[w][lane + 64 * e] = o[e];
    if (lane == 0) {
        s_m[w] = M;
        s_l[w] = L;
    }
    __syncthreads();
    if (page_named(p.pages, entry) < 0) {
        if (tid < D) ((T *)p.out)[head * D + tid] = (T)NAN;
        if (p.lse && tid == 0) p.lse[head] = NAN;
        if (p.len_out && h == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    if (tid < D) {
        float top = -INFINITY, sum = 0.0f, out = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) top = fmaxf(top, s_m[x]);
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float f = s_m[x] == top ? 1.0f : __builtin_amdgcn_exp2f(s_m[x] - top);
            sum += s_l[x] * f;
            out += s_o[x][tid] * f;
        }
        ((T *)p.out)[head * D + tid] = (T)(out / sum);
        if (tid == 0) {
            if (p.lse) {
                const FusionBias fb = fusion_bias(p.gate[s * p.gss + h * p.gsh], p.clamp > 0.0f);
                p.lse[head] = (top + __log2f(sum)) * kLn2 + fb.lse_shift;
            }
            if (p.len_out && h == 0) p.len_out[s] = t + 1;
        }
    }
}

template <typename T, int D>
hipError_t launch_join_d(const PagedStepParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)(p.S * p.H));
    return p.parts > 32 ? launch_kernel(join_kernel<T, D, 16>, grid, dim3(1024), stream, p)
                        : launch_kernel(join_kernel<T, D, 4>, grid, dim3(256), stream, p);
}

template <typename T>
hipError_t launch_join(const PagedStepParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_join_d<T, 64>(p, stream) : launch_join_d<T, 128>(p, stream);
}

}  // namespace

// Where a few (s, key head) can have long windows, these are split, by the lengths that
// they turn out to have (range_len), which balances sequences of unlike lengths too.  A
// split costs the join's launch, 4 us.  us, whole and split, bf16, D = 128, four query
// heads each: 8 (s, key head) of 512 rows 10.6 and 12.6, of 1024 14.7 and 12.8, of 2040 22.1
// and 12.0; 64 of 1024 17.7 and 17.9, of 2040 27.5 and 20.9; 128 of 1024 19.0 and 22.3, of
// 2000 to 4095 51.5 and 41.8; 256 of 1024 27.0 and 32.0, of 2040 45.2 and 50.6.  Ranges of
// 8 windows of 65536: of 256 rows 55.9, 512 51.9, 1024 50.3, 2048 51.7.  At most some 4096
// work-groups (those of ranges that a window has not end at once) for each group of query
// heads of a key head (16, of float32 pages 8), and fewer than 2^32 threads.
void plan_decode_paged(PagedStepParams &p) {
    const int64_t n = (int64_t)p.S * p.Hk, rows = longest_window(p);
    p.parts = 0;
    if (n >= 4096 || rows <= (n <= 16 ? 768 : n <= 192 ? 1024 : 2048)) return;
    const int64_t parts = std::min({std::max(768 / n + 1, (rows + 1023) / 1024), (rows + 127) / 128, 4096 / n,
                                    (int64_t)(1 << 23) / ((int64_t)p.S * p.H)});
    if (parts > 1) p.parts = (int)parts;
}

hipError_t launch_decode_paged(const PagedStepParams &p, bool bf16, hipStream_t stream) {
    const bool tiles = bf16 || p.pages.k_exp;
    const hipError_t e = tiles ? launch_decode_paged_tiles(p, bf16, stream) : launch_decode_paged_f32(p, stream);
    if (e != hipSuccess || p.parts == 0) return e;
    return bf16 ? launch_join<__bf16>(p, stream) : launch_join<float>(p, stream);
}

}  // namespace pi_attn
