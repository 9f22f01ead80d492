/* Calls the oracle's norm, rotation and attention on small and edge-case inputs,
 * every buffer exactly as large as documented, for a build with sanitizers. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

void oracle_norm_rope(const void *x, int is_bf16, int32_t T, int32_t n, int32_t hd,
                      const int32_t *pos, const void *weight, double eps, const double *inv_freq,
                      int32_t rot, int32_t pairs, double *out);
void oracle_attend(const uint16_t *q, int32_t T, int32_t n_q, int32_t hd, const int32_t *cu,
                   const int32_t *kv_len, int32_t R, const double *k, const double *v,
                   const int32_t *pages, int32_t n_pages, int32_t max_pages, int32_t page_size,
                   int32_t n_kv, double scale, int32_t window, double *out, double *lse,
                   double *mag, double *big);

#define NEW(type, n) ((type *)calloc((size_t)(n), sizeof(type)))

static void norms(int32_t T, int32_t n, int32_t hd, int32_t rot, int bf16) {
    float *xf = NEW(float, T * n * hd), *wf = NEW(float, hd);
    uint16_t *xb = NEW(uint16_t, T * n * hd), *wb = NEW(uint16_t, hd);
    int32_t *pos = NEW(int32_t, T);
    double *f = NEW(double, rot / 2 + 1), *out = NEW(double, T * n * hd);
    for (int i = 0; i < T * n * hd; ++i) { xf[i] = (float)(i % 17) - 8.0f; xb[i] = 0x3F80 + i % 64; }
    for (int i = 0; i < hd; ++i) { wf[i] = 1.0f; wb[i] = 0x3F80; }
    for (int t = 0; t < T; ++t) pos[t] = t == 1 ? -1 : t == 2 ? INT32_MAX : t;
    for (int i = 0; i < rot / 2; ++i) f[i] = pow(1e4, -i / 8.0);
    for (int pairs = 0; pairs < 2; ++pairs) {
        oracle_norm_rope(bf16 ? (void *)xb : (void *)xf, bf16, T, n, hd, pos,
                         bf16 ? (void *)wb : (void *)wf, 1e-6, rot ? f : NULL, rot, pairs, out);
        oracle_norm_rope(bf16 ? (void *)xb : (void *)xf, bf16, T, n, hd, pos, NULL, 0.0,
                         rot ? f : NULL, rot, pairs, out);
    }
    free(xf); free(wf); free(xb); free(wb); free(pos); free(f); free(out);
}

static void attends(int32_t window) {
    /* spans of one, no and several tokens, without keys, with fewer keys than tokens,
       up to a full table, and a page that is not there */
    const int32_t R = 6, hd = 16, n_q = 4, n_kv = 2, ps = 16, max_pages = 3, n_pages = 4;
    const int32_t cu[7] = {0, 1, 1, 4, 6, 7, 12}, len[6] = {1, 9, 0, 1, 33, 48}, T = 13;
    int32_t *pages = NEW(int32_t, R * max_pages);
    uint16_t *q = NEW(uint16_t, T * n_q * hd);
    double *k = NEW(double, n_pages * n_kv * ps * hd), *v = NEW(double, n_pages * n_kv * ps * hd);
    double *out = NEW(double, T * n_q * hd), *mag = NEW(double, T * n_q * hd);
    double *lse = NEW(double, n_q * T), *big = NEW(double, n_q * T);
    for (int i = 0; i < R * max_pages; ++i) pages[i] = i % n_pages;
    pages[4 * max_pages + 1] = n_pages;
    pages[5 * max_pages + 2] = -1;
    for (int i = 0; i < T * n_q * hd; ++i) q[i] = 0x3F00 + i % 128;
    for (int i = 0; i < n_pages * n_kv * ps * hd; ++i) { k[i] = i % 13 - 6; v[i] = i % 7 - 3; }
    oracle_attend(q, T, n_q, hd, cu, len, R, k, v, pages, n_pages, max_pages, ps, n_kv, 0.25, window,
                  out, lse, mag, big);
    for (int i = 0; i < n_q * hd; ++i)
        if (out[12 * n_q * hd + i] != 0.0) abort(); /* outside every span */
    free(pages); free(q); free(k); free(v); free(out); free(mag); free(lse); free(big);
}

int main(void) {
    norms(1, 1, 16, 0, 1);
    norms(5, 3, 48, 32, 1);
    norms(4, 2, 256, 256, 0);
    for (int w = 0; w < 40; w += 13) attends(w);
    printf("sanitized attention oracle ok\n");
    return 0;
}
