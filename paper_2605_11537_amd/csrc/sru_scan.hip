// sru_scan and its gradient: the recurrence of an SRU layer over pre-activations that lie in memory.
#include "scalar_math.h"

namespace moe {

constexpr int SCAN_THREADS = 64;
constexpr int SCAN_STEPS = 16;         // steps per saved state

template <class T, bool HIGHWAY>
__global__ __launch_bounds__(SCAN_THREADS) void sru_scan_kernel(const T *__restrict__ u, const T *__restrict__ x,
                                                                const float *__restrict__ b_f, const float *__restrict__ b_r,
                                                                const float *c0, const int32_t *__restrict__ lengths, int L, int H,
                                                                int blocks, T *__restrict__ h, float *c_last, float *__restrict__ states)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    const int b = blockIdx.x / blocks, ch = blockIdx.x % blocks * SCAN_THREADS + threadIdx.x;
    if (ch >= H) return;
    const int n = lengths ? min(max(lengths[b], 0), L) : L;
    const float bf = b_f ? b_f[ch] : 0.f, br = b_r ? b_r[ch] : 0.f;
    const int saved = (L + SCAN_STEPS - 1) / SCAN_STEPS;
    float c = c0 ? c0[(size_t)b * H + ch] : 0.f;
    for (int t = 0; t < L; ++t) {
        const size_t row = (size_t)b * L + t;
        if (states && t % SCAN_STEPS == 0) states[((size_t)b * saved + t / SCAN_STEPS) * H + ch] = c;
        if (t >= n) {
            store_value(h + row * H + ch, 0.f);
            continue;
        }
        const T *ur = u + row * K * H + ch;
        const float z = value_of(ur[0]), w = HIGHWAY ? value_of(x[row * H + ch]) : value_of(ur[(size_t)(K - 1) * H]);
        float f, fr, r, rr, slope;
        gate_of<PRECISE>(value_of(ur[H]) + bf, f, fr);
        gate_of<PRECISE>(value_of(ur[2 * (size_t)H]) + br, r, rr);
        c = fmaf(f, c, fr * z);
        store_value(h + row * H + ch, fmaf(r, tanh_of<PRECISE>(c, slope), rr * w));
    }
    if (c_last) c_last[(size_t)b * H + ch] = c;
}

template <class T, bool HIGHWAY>
__global__ __launch_bounds__(SCAN_THREADS) void sru_scan_backward_kernel(
    const T *__restrict__ dh, const float *dc_last, const T *__restrict__ u, const T *__restrict__ x, const float *__restrict__ b_f,
    const float *__restrict__ b_r, const float *__restrict__ states, const int32_t *__restrict__ lengths, int L, int H, int blocks,
    T *__restrict__ du, T *__restrict__ dx, float *__restrict__ db, float *dc0)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    const int b = blockIdx.x / blocks, ch = blockIdx.x % blocks * SCAN_THREADS + threadIdx.x;
    if (ch >= H) return;
    const int n = lengths ? min(max(lengths[b], 0), L) : L;
    const float bf = b_f ? b_f[ch] : 0.f, br = b_r ? b_r[ch] : 0.f;
    const int saved = (L + SCAN_STEPS - 1) / SCAN_STEPS;
    float dc = dc_last ? dc_last[(size_t)b * H + ch] : 0.f, sum_f = 0.f, sum_r = 0.f;
    for (int part = saved - 1; part >= 0; --part) {
        const int t0 = part * SCAN_STEPS, t1 = min(L, t0 + SCAN_STEPS);
        float before[SCAN_STEPS];
        float c = states[((size_t)b * saved + part) * H + ch];
#pragma unroll
        for (int i = 0; i < SCAN_STEPS; ++i) {
            before[i] = c;
            if (t0 + i >= n) continue;
            const T *ur = u + ((size_t)b * L + t0 + i) * K * H + ch;
            float f, fr;
            gate_of<PRECISE>(value_of(ur[H]) + bf, f, fr);
            c = fmaf(f, c, fr * value_of(ur[0]));
        }
#pragma unroll
        for (int i = SCAN_STEPS - 1; i >= 0; --i) {
            const int t = t0 + i;
            if (t >= t1) continue;
            const size_t row = (size_t)b * L + t;
            T *dr = du + row * K * H + ch, *dw = HIGHWAY ? dx + row * H + ch : dr + (size_t)(K - 1) * H;
            if (t >= n) {
                store_value(dr, 0.f), store_value(dr + H, 0.f), store_value(dr + 2 * (size_t)H, 0.f), store_value(dw, 0.f);
                continue;
            }
            const T *ur = u + row * K * H + ch;
            const float z = value_of(ur[0]), w = HIGHWAY ? value_of(x[row * H + ch]) : value_of(ur[(size_t)(K - 1) * H]);
            float f, fr, r, rr, slope;
            gate_of<PRECISE>(value_of(ur[H]) + bf, f, fr);
            gate_of<PRECISE>(value_of(ur[2 * (size_t)H]) + br, r, rr);
            const float g = tanh_of<PRECISE>(fmaf(f, before[i], fr * z), slope), d = value_of(dh[row * H + ch]);
            const float full = fmaf(d * r, slope, dc);
            const float d_f = full * (before[i] - z) * (f * fr), d_r = d * (g - w) * (r * rr);
            store_value(dw, d * rr);
            store_value(dr, full * fr);
            store_value(dr + H, d_f);
            store_value(dr + 2 * (size_t)H, d_r);
            sum_f += d_f;
            sum_r += d_r;
            dc = full * f;
        }
    }
    if (dc0) dc0[(size_t)b * H + ch] = dc;
    db[(size_t)b * 2 * H + ch] = sum_f;
    db[((size_t)b * 2 + 1) * H + ch] = sum_r;
}

// db_f and db_r: the parts' sums in their order
__global__ __launch_bounds__(SCAN_THREADS) void sru_scan_bias_kernel(const float *__restrict__ db, int parts, int H, float *__restrict__ db_f,
                                                                     float *__restrict__ db_r)
{
    const int ch = blockIdx.x * SCAN_THREADS + threadIdx.x;
    if (ch >= 2 * H) return;
    float *out = ch < H ? db_f : db_r;
    if (!out) return;
    float sum = 0.f;
    for (int p = 0; p < parts; ++p) sum += db[(size_t)p * 2 * H + ch];
    out[ch < H ? ch : ch - H] = sum;
}

static int scan_check(const char *who, int B, int L, int H, int n_blocks, int dtype, const void *x)
{
    MOE_REQUIRE(B >= 0 && L >= 0 && H > 0, MOE_ERR_INVALID_ARG, "%s: B=%d L=%d H=%d out of range", who, B, L, H);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE(n_blocks == 3 || n_blocks == 4, MOE_ERR_INVALID_ARG, "%s: n_blocks=%d (3 with x, 4 without)", who, n_blocks);
    MOE_REQUIRE(n_blocks == 3 || !x, MOE_ERR_INVALID_ARG, "%s: x given beside a fourth block", who);
    MOE_REQUIRE((long long)B * ((H + SCAN_THREADS - 1) / SCAN_THREADS) < (1 << 26), MOE_ERR_UNSUPPORTED, "%s: B=%d H=%d too large", who, B, H);
    return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t sru_scan_states_bytes(int B, int L, int H)
{
    if (B <= 0 || L <= 0 || H <= 0) return 0;
    return (size_t)B * ((L + SCAN_STEPS - 1) / SCAN_STEPS) * H * sizeof(float);
}

extern "C" size_t sru_scan_workspace_bytes(int B, int L, int H, int dtype)
{
    (void)B, (void)L, (void)H, (void)dtype;
    return 0;
}

extern "C" size_t sru_scan_backward_workspace_bytes(int B, int L, int H, int dtype)
{
    (void)L, (void)dtype;
    if (B <= 0 || H <= 0) return 0;
    return (size_t)B * 2 * H * sizeof(float);
}

extern "C" int sru_scan(const void *u, const void *x, const float *b_f, const float *b_r, const float *c0, const int32_t *lengths, int B,
                        int L, int H, int n_blocks, int dtype, void *h, float *c_last, void *states, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = scan_check("sru_scan", B, L, H, n_blocks, dtype, x);
    if (rc != MOE_OK || B == 0) return rc;
    if (L > 0) {
        MOE_REQUIRE(u && h && (n_blocks == 4 || x), MOE_ERR_INVALID_ARG, "sru_scan: null pointer");
        MOE_REQUIRE(h != u && h != x, MOE_ERR_INVALID_ARG, "sru_scan: h aliases an input");
        MOE_REQUIRE(aligned16(u) && aligned16(x) && aligned16(h) && aligned16(states), MOE_ERR_INVALID_ARG, "sru_scan: tensor misaligned");
    }
    const int blocks = (H + SCAN_THREADS - 1) / SCAN_THREADS;
    hipStream_t st = (hipStream_t)stream;
#define MOE_SCAN(T, HW)                                                                                                          \
    hipLaunchKernelGGL((sru_scan_kernel<T, HW>), dim3(B *blocks), dim3(SCAN_THREADS), 0, st, (const T *)u, (const T *)x, b_f, b_r, c0, \
                       lengths, L, H, blocks, (T *)h, c_last, (float *)states)
    if (dtype == MOE_BF16) {
        if (n_blocks == 3) MOE_SCAN(bf16_t, true);
        else MOE_SCAN(bf16_t, false);
    } else {
        if (n_blocks == 3) MOE_SCAN(float, true);
        else MOE_SCAN(float, false);
    }
#undef MOE_SCAN
    MOE_CHECK_LAUNCH("sru_scan");
    return MOE_OK;
}

extern "C" int sru_scan_backward(const void *dh, const float *dc_last, const void *u, const void *x, const float *b_f, const float *b_r,
                                 const void *states, const int32_t *lengths, int B, int L, int H, int n_blocks, int dtype, void *du,
                                 void *dx, float *db_f, float *db_r, float *dc0, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = scan_check("sru_scan_backward", B, L, H, n_blocks, dtype, x);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(n_blocks == 3 || !dx, MOE_ERR_INVALID_ARG, "sru_scan_backward: dx given beside a fourth block");
    if (B > 0 && L > 0) {
        MOE_REQUIRE(dh && u && states && du && (n_blocks == 4 || (x && dx)), MOE_ERR_INVALID_ARG, "sru_scan_backward: null pointer");
        MOE_REQUIRE(du != u && du != x && du != dh && (!dx || (dx != u && dx != x && dx != dh && dx != du)), MOE_ERR_INVALID_ARG,
                    "sru_scan_backward: an output aliases another tensor");
        MOE_REQUIRE(aligned16(dh) && aligned16(u) && aligned16(x) && aligned16(states) && aligned16(du) && aligned16(dx), MOE_ERR_INVALID_ARG,
                    "sru_scan_backward: tensor misaligned");
    }
    const size_t need = sru_scan_backward_workspace_bytes(B, L, H, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE,
                "sru_scan_backward: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, need);
    const int blocks = (H + SCAN_THREADS - 1) / SCAN_THREADS;
    hipStream_t st = (hipStream_t)stream;
#define MOE_SCAN(T, HW)                                                                                                                   \
    hipLaunchKernelGGL((sru_scan_backward_kernel<T, HW>), dim3(B *blocks), dim3(SCAN_THREADS), 0, st, (const T *)dh, dc_last, (const T *)u, \
                       (const T *)x, b_f, b_r, (const float *)states, lengths, L, H, blocks, (T *)du, (T *)dx, (float *)ws, dc0)
    if (B > 0) {
        if (dtype == MOE_BF16) {
            if (n_blocks == 3) MOE_SCAN(bf16_t, true);
            else MOE_SCAN(bf16_t, false);
        } else {
            if (n_blocks == 3) MOE_SCAN(float, true);
            else MOE_SCAN(float, false);
        }
        MOE_CHECK_LAUNCH("sru_scan_backward");
    }
#undef MOE_SCAN
    if (db_f || db_r) {
        hipLaunchKernelGGL(sru_scan_bias_kernel, dim3((2 * H + SCAN_THREADS - 1) / SCAN_THREADS), dim3(SCAN_THREADS), 0, st, (const float *)ws,
                           B, H, db_f, db_r);
        MOE_CHECK_LAUNCH("sru_scan_backward");
    }
    return MOE_OK;
}
