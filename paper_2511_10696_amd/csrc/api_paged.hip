// api_paged.hip -- the C ABI of the rotary positions and of the paged caches:
// argument validation and dispatch, as in api.hip.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/pi_attn.h"
#include "checks.h"
#include "paged.h"

using namespace pi_attn;

namespace {

bool strides_ok(int es, int64_t a, int64_t b, int64_t c) { return stride16(a, es) && stride16(b, es) && stride16(c, es); }

// Rows that a call writes lie apart: by rising stride, the dimensions of more than one row are
// nested in each other, as any order of them in memory and any slice of it is.
bool apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t D) {
    struct Dim {
        int64_t n, s;
    } dims[3] = {{n0, s0}, {n1, s1}, {n2, s2}};
    std::sort(dims, dims + 3, [](const Dim &a, const Dim &b) { return a.s < b.s; });
    int64_t least = D;
    for (const Dim &d : dims) {
        if (d.n <= 1) continue;
        if (d.s < least) return false;
        least = d.n > INT64_MAX / d.s ? INT64_MAX : d.n * d.s;
    }
    return true;
}

// The rotation of rows of D elements; freq == nullptr or no pairs: none.
int check_rotary(const float *freq, int32_t n0, int32_t n1, int32_t n2, const int32_t *pos, int64_t psa, int64_t psb,
                 int64_t psn, int32_t D, Rotary &r) {
    r = Rotary{};
    if (!freq) return PI_ATTN_OK;
    if (n0 < 0 || n1 < 0 || n2 < 0 || (int64_t)n0 + n1 + n2 > D / 2) return PI_ATTN_EINVAL;
    if (!aligned4(freq) || (pos && !aligned4(pos)) || psa < 0 || psb < 0 || psn < 0) return PI_ATTN_EINVAL;
    if (n0 + n1 + n2 == 0) return PI_ATTN_OK;
    r.freq = freq;
    r.end0 = n0;
    r.end1 = n0 + n1;
    r.pairs = n0 + n1 + n2;
    r.pos = pos;
    r.psa = psa;
    r.psb = psb;
    r.psn = psn;
    return PI_ATTN_OK;
}

// Sizes of a paged cache that the kernels index with 32 bits: positions, with a
// tile's rows to spare.
int check_page_sizes(int32_t n_pages, int32_t page, int32_t max_pages) {
    if (n_pages < 1 || page < 1 || max_pages < 1) return PI_ATTN_EINVAL;
    return (int64_t)page * max_pages <= INT32_MAX - 4096 ? PI_ATTN_OK : PI_ATTN_EUNSUPPORTED;
}

// A paged cache whose sizes are valid.
int check_pages(int32_t n_pages, int32_t page, int32_t max_pages, const int32_t *table, void *k, void *v, uint8_t *k_exp,
                uint8_t *v_exp, Pages &g) {
    if (!table || !k || !v || !aligned4(table) || !aligned16(k) || !aligned16(v)) return PI_ATTN_EINVAL;
    if ((k_exp != nullptr) != (v_exp != nullptr)) return PI_ATTN_EINVAL;
    g.n_pages = n_pages;
    g.page = page;
    g.max_pages = max_pages;
    g.by_page = Divisor(page);
    g.table = table;
    g.k = k;
    g.v = v;
    g.k_exp = k_exp;
    g.v_exp = v_exp;
    return PI_ATTN_OK;
}

// Both directions between rows in the working type and a paged cache.
int paged_rows(bool store, int32_t dtype, int32_t S, int32_t Hk, int32_t D, int32_t n, int32_t n_pages, int32_t page,
               int32_t max_pages, void *k, void *v, int64_t sb, int64_t sh, int64_t sn, const int32_t *start,
               const int32_t *count, const int32_t *table, void *k_pages, void *v_pages, uint8_t *k_exp, uint8_t *v_exp,
               const float *freq, int32_t n0, int32_t n1, int32_t n2, const int32_t *pos, int64_t psa, int64_t psb,
               int64_t psn, void *stream) {
    const int es = elem_size(dtype);
    if (es == 0) return PI_ATTN_EUNSUPPORTED;
    if (S < 0 || Hk < 0 || n < 0) return PI_ATTN_EINVAL;
    if (D != 64 && D != 128) return PI_ATTN_EUNSUPPORTED;
    PagedRowsParams p{};
    int status = check_page_sizes(n_pages, page, max_pages);
    if (status != PI_ATTN_OK) return status;
    status = check_rotary(freq, n0, n1, n2, pos, psa, psb, psn, D, p.r);
    if (status != PI_ATTN_OK) return status;
    if ((int64_t)S * Hk >= kMaxRows || (int64_t)S * n >= kMaxRows || (int64_t)S * Hk * n >= kMaxRows) return PI_ATTN_EINVAL;
    if ((int64_t)S * Hk * n == 0) return PI_ATTN_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v) || !strides_ok(es, sb, sh, sn)) return PI_ATTN_EINVAL;
    if ((start && !aligned4(start)) || (count && !aligned4(count))) return PI_ATTN_EINVAL;
    if (!store && (k == v || !apart(S, sb, Hk, sh, n, sn, D))) return PI_ATTN_EINVAL;
    status = check_pages(n_pages, page, max_pages, table, k_pages, v_pages, k_exp, v_exp, p.pages);
    if (status != PI_ATTN_OK) return status;
    p.S = S; p.Hk = Hk; p.n = n; p.D = D;
    p.k = k; p.v = v; p.sb = sb; p.sh = sh; p.sn = sn;
    p.start = start; p.count = count;
    p.rows = (uint32_t)((int64_t)S * n);
    p.by_n = Divisor(n);
    return from_hip(launch_paged_rows(p, store, dtype == PI_ATTN_BF16, (hipStream_t)stream));
}

// The sizes of a paged step.
int check_paged_step(int32_t dtype, int32_t S, int32_t H, int32_t Hk, int32_t D, int32_t n_pages, int32_t page,
                     int32_t max_pages, int32_t k, PagedStepParams &p, bool &empty) {
    empty = false;
    if (elem_size(dtype) == 0) return PI_ATTN_EUNSUPPORTED;
    if (S < 0 || H < 0 || Hk < 0 || k < 0 || (Hk == 0) != (H == 0) || (Hk > 0 && H % Hk != 0)) return PI_ATTN_EINVAL;
    if (D != 64 && D != 128) return PI_ATTN_EUNSUPPORTED;
    const int status = check_page_sizes(n_pages, page, max_pages);
    if (status != PI_ATTN_OK) return status;
    empty = S == 0 || H == 0;
    // a work-group of 256 threads for each (s, h): fewer than 2^32 threads; rows of
    // the pool are counted in 32 bits
    if ((int64_t)S * H >= 1 << 24 || (int64_t)n_pages * page >= kMaxRows || (int64_t)n_pages * page * Hk >= kMaxRows)
        return PI_ATTN_EUNSUPPORTED;
    p.S = S; p.H = H; p.Hk = Hk; p.D = D; p.k = k;
    p.pages.n_pages = n_pages;
    p.pages.page = page;
    p.pages.max_pages = max_pages;
    if (!empty) plan_decode_paged(p);
    return PI_ATTN_OK;
}

}  // namespace

extern "C" {

int pi_attn_rotate(int32_t dtype, int32_t out_dtype, int32_t B, int32_t H, int32_t Hk, int32_t N, int32_t D, int32_t back,
                   const void *q, int64_t qsb, int64_t qsh, int64_t qsn, const void *k, int64_t ksb, int64_t ksh,
                   int64_t ksn, const int32_t *pos, int64_t psa, int64_t psb, int64_t psn, const float *freq, int32_t n0,
                   int32_t n1, int32_t n2, void *q_out, int64_t oqsb, int64_t oqsh, int64_t oqsn, void *k_out,
                   int64_t oksb, int64_t oksh, int64_t oksn, void *stream) {
    const int es = elem_size(dtype), eo = elem_size(out_dtype);
    if (es == 0 || eo == 0) return PI_ATTN_EUNSUPPORTED;
    if (B < 0 || H < 0 || Hk < 0 || N < 0) return PI_ATTN_EINVAL;
    if (D != 64 && D != 128) return PI_ATTN_EUNSUPPORTED;
    RotateParams p{};
    const int status = check_rotary(freq, n0, n1, n2, pos, psa, psb, psn, D, p.r);
    if (status != PI_ATTN_OK) return status;
    const int64_t heads = (int64_t)H + Hk;
    if ((int64_t)B * N >= kMaxRows || heads >= kMaxRows || (int64_t)B * N * heads >= kMaxRows) return PI_ATTN_EINVAL;
    if ((int64_t)B * N * heads == 0) return PI_ATTN_OK;
    if (H > 0) {
        if (!q || !q_out || !aligned16(q) || !aligned16(q_out)) return PI_ATTN_EINVAL;
        if (!strides_ok(es, qsb, qsh, qsn) || !strides_ok(eo, oqsb, oqsh, oqsn)) return PI_ATTN_EINVAL;
        if (!apart(B, oqsb, H, oqsh, N, oqsn, D)) return PI_ATTN_EINVAL;
        if (q == q_out && (es != eo || qsb != oqsb || qsh != oqsh || qsn != oqsn)) return PI_ATTN_EINVAL;
    }
    if (Hk > 0) {
        if (!k || !k_out || !aligned16(k) || !aligned16(k_out)) return PI_ATTN_EINVAL;
        if (!strides_ok(es, ksb, ksh, ksn) || !strides_ok(eo, oksb, oksh, oksn)) return PI_ATTN_EINVAL;
        if (!apart(B, oksb, Hk, oksh, N, oksn, D)) return PI_ATTN_EINVAL;
        if (k == k_out && (es != eo || ksb != oksb || ksh != oksh || ksn != oksn)) return PI_ATTN_EINVAL;
    }
    if (H > 0 && Hk > 0 && (q_out == k_out || q_out == k || k_out == q)) return PI_ATTN_EINVAL;
    p.B = B; p.H = H; p.Hk = Hk; p.N = N; p.D = D;
    p.q = q; p.k = k; p.q_out = q_out; p.k_out = k_out;
    p.qsb = qsb; p.qsh = qsh; p.qsn = qsn; p.ksb = ksb; p.ksh = ksh; p.ksn = ksn;
    p.oqsb = oqsb; p.oqsh = oqsh; p.oqsn = oqsn; p.oksb = oksb; p.oksh = oksh; p.oksn = oksn;
    p.back = back != 0;
    p.rows = (uint32_t)((int64_t)B * N);
    p.by_n = Divisor(N);
    return from_hip(launch_rotate(p, dtype == PI_ATTN_BF16, out_dtype == PI_ATTN_BF16, (hipStream_t)stream));
}

int pi_attn_paged_store(int32_t dtype, int32_t S, int32_t Hk, int32_t D, int32_t n, int32_t n_pages, int32_t page,
                        int32_t max_pages, const void *k, const void *v, int64_t sb, int64_t sh, int64_t sn,
                        const int32_t *start, const int32_t *count, const int32_t *table, void *k_pages, void *v_pages,
                        uint8_t *k_exp, uint8_t *v_exp, const float *freq, int32_t n0, int32_t n1, int32_t n2,
                        const int32_t *pos, int64_t psa, int64_t psb, int64_t psn, void *stream) {
    return paged_rows(true, dtype, S, Hk, D, n, n_pages, page, max_pages, const_cast<void *>(k), const_cast<void *>(v), sb,
                      sh, sn, start, count, table, k_pages, v_pages, k_exp, v_exp, freq, n0, n1, n2, pos, psa, psb, psn,
                      stream);
}

int pi_attn_paged_load(int32_t dtype, int32_t S, int32_t Hk, int32_t D, int32_t n, int32_t n_pages, int32_t page,
                       int32_t max_pages, const void *k_pages, const void *v_pages, const uint8_t *k_exp,
                       const uint8_t *v_exp, const int32_t *start, const int32_t *count, const int32_t *table, void *k,
                       void *v, int64_t sb, int64_t sh, int64_t sn, void *stream) {
    return paged_rows(false, dtype, S, Hk, D, n, n_pages, page, max_pages, k, v, sb, sh, sn, start, count, table,
                      const_cast<void *>(k_pages), const_cast<void *>(v_pages), const_cast<uint8_t *>(k_exp),
                      const_cast<uint8_t *>(v_exp), nullptr, 0, 0, 0, nullptr, 0, 0, 0, stream);
}

int64_t pi_attn_paged_workspace(int32_t dtype, int32_t S, int32_t H, int32_t Hk, int32_t D, int32_t page,
                                int32_t max_pages, int32_t k) {
    PagedStepParams p{};
    bool empty;
    if (check_paged_step(dtype, S, H, Hk, D, 1, page, max_pages, k, p, empty) != PI_ATTN_OK) return -1;
    return (int64_t)p.parts * S * H * (D + 2);
}

int pi_attn_decode_step_paged(int32_t dtype, int32_t S, int32_t H, int32_t Hk, int32_t D, int32_t n_pages, int32_t page,
                              int32_t max_pages, int32_t k, int32_t pi, const int32_t *len_in, int32_t *len_out,
                              const void *q_new, const void *k_new, const void *v_new, const int32_t *table,
                              void *k_pages, void *v_pages, uint8_t *k_exp, uint8_t *v_exp, const float *freq, int32_t n0,
                              int32_t n1, int32_t n2, const int32_t *pos, int64_t psa, int64_t pss, const float *gate,
                              int64_t gss, int64_t gsh, float scale, float logit_clamp, void *out, float *lse,
                              float *work, void *stream) {
    PagedStepParams p{};
    bool empty;
    int status = check_paged_step(dtype, S, H, Hk, D, n_pages, page, max_pages, k, p, empty);
    if (status != PI_ATTN_OK) return status;
    if (pi < 0 || !isfinite(scale) || scale <= 0.0f || isnan(logit_clamp)) return PI_ATTN_EINVAL;
    status = check_rotary(freq, n0, n1, n2, pos, psa, pss, 0, D, p.r);
    if (status != PI_ATTN_OK || empty) return status;
    if (!len_in || !q_new || !k_new || !v_new || !gate || !out) return PI_ATTN_EINVAL;
    if (len_out) {   // other work-groups of the step still read len_in
        const uintptr_t a = reinterpret_cast<uintptr_t>(len_in), b = reinterpret_cast<uintptr_t>(len_out);
        const uintptr_t bytes = (uintptr_t)S * sizeof(int32_t);
        if (a < b + bytes && b < a + bytes) return PI_ATTN_EINVAL;
    }
    if (!aligned4(len_in) || (len_out && !aligned4(len_out))) return PI_ATTN_EINVAL;
    if (!aligned16(q_new) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out)) return PI_ATTN_EINVAL;
    if (!aligned4(gate) || gss < 0 || gsh < 0 || (lse && !aligned4(lse))) return PI_ATTN_EINVAL;
    status = check_pages(n_pages, page, max_pages, table, k_pages, v_pages, k_exp, v_exp, p.pages);
    if (status != PI_ATTN_OK) return status;
    if (p.parts && (!work || !aligned16(work))) return PI_ATTN_EINVAL;
    p.pi = pi;
    p.len_in = len_in; p.len_out = len_out;
    p.q_new = q_new; p.k_new = k_new; p.v_new = v_new;
    p.gate = gate; p.gss = gss; p.gsh = gsh;
    p.scale = scale;
    p.clamp = logit_clamp > 0.0f ? logit_clamp : 0.0f;
    p.out = out; p.lse = lse;
    p.part_o = work;
    p.part_ml = p.parts ? work + (int64_t)p.parts * S * H * D : nullptr;
    return from_hip(launch_decode_paged(p, dtype == PI_ATTN_BF16, (hipStream_t)stream));
}

}  // extern "C"
