// One layer in the structured-only form with bias, activation and residual behind the product, and a gated block (gfx950):
//     z[b][s] = bias[a(s)] + sum_j Wd[s][j] x[b][j],   y[b][a(s)] = act(z[b][s]) + r[b][a(s)],   other columns c: act(bias[c]) + r[b][c]
//     h[b][c] = act(bg[c] + sum_j Wg[c][j] x[b][j]) * (bu[c] + sum_j Wu[c][j] x[b][j])
// The gated block is one product over both weight matrices' rows: a workgroup's tile holds the same rows of both, each wavefront the gate's sums and the
// up-projection's of the same neurons, so that they meet in the epilogue and neither projection goes to memory (unless the caller keeps them for
// the backward pass).
#include "dense_tile.h"

namespace srigl {

// Expected time (us) of a product in a tile and `parts` parts of K: rounds of workgroups over the compute units, each a fixed part and a part per 1000 elements of K
// (less where a workgroup has its compute unit to itself); the parts' sums are written and read and joined by a second launch.
struct DenseModel { int bm, bn; float fixed, round, per_k, alone; int slots; };
static const DenseModel kDenseBf16[] = {{64, 64, 2.8f, 1.1f, 5.6f, 0.65f, 512}, {128, 128, 3.1f, 3.0f, 9.3f, 1.0f, 256}, {256, 128, 1.6f, 4.7f, 10.5f, 1.0f, 256}, {256, 256, 0.7f, 7.0f, 20.2f, 1.0f, 256}};
static const DenseModel kDenseF32[] = {{64, 64, 2.1f, 1.0f, 38.0f, 0.5f, 512}, {128, 128, 2.1f, 2.0f, 70.0f, 1.0f, 256}};
static const DenseModel kPairBf16 = {64, 128, 2.0f, 3.0f, 5.0f, 1.0f, 256}, kPairF32 = {64, 128, 2.1f, 2.0f, 38.0f, 1.0f, 256};
constexpr float kJoinUs = 2.5f, kPartUs = 1.8e-6f;   // a second launch; a part's sum written and read

// direct: rows are multiples of 16 bytes (a choice by sizes, so that the workspace does not depend on addresses)
DensePlan plan_dense(int M, int N, int stages, bool f32, bool pair, bool direct) {
    if (M <= 0 || N <= 0) return {kTileS, 1};
    struct Key { int32_t M, N, stages, form; };
    static thread_local DecisionCache<Key, DensePlan, 64> cache;
    return cache.get(Key{M, N, stages, f32 + 2 * pair + 4 * direct}, [&] {
        DensePlan best{kTileS, 1};
        double best_us = 0.0;
        const double d = 1e-3 * stages * (f32 ? 32 : 64), sums = (double)M * N * (pair ? 2 : 1);
        for (int t = 0; t < (f32 || !direct ? 2 : 4); ++t) {
            const DenseModel& m = pair && t == kTileS ? (f32 ? kPairF32 : kPairBf16) : (f32 ? kDenseF32 : kDenseBf16)[t];
            const long long cols = pair ? m.bn / 2 : m.bn, tiles = ((M + m.bm - 1ll) / m.bm) * ((N + cols - 1) / cols), padded = (tiles + kXcds - 1) / kXcds * kXcds;
            for (int parts = 1; parts <= 16; ++parts) {
                if (parts > 1 && (parts * 2 > stages || padded * parts > m.slots)) break;   // two stages to a part; parts side by side
                const double groups = (double)(parts > 1 ? padded * parts : tiles);
                const double us = m.fixed + std::ceil(groups / m.slots) * (m.round + (groups <= 256 ? m.alone : 1.0f) * m.per_k * d / parts) +
                                  (parts > 1 ? kJoinUs + kPartUs * parts * sums : 0.0);
                if (best_us == 0.0 || us < best_us) best = {t, parts}, best_us = us;
            }
        }
        return best;
    });
}

template <typename T, typename TY>
struct LinearOut {
    static constexpr bool kListed = true;
    const int32_t* active;
    int n_active;
    const float* bias;
    const TY* residual;
    int d_out;
    TY* y;
    T* z;      // pre-activations [B][n_active], or nullptr
    int act;
    float b[8];    // of the thread's columns

    template <int V> __device__ void start(int s, int valid) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            b[q] = 0.0f;
            if (bias && q < valid) {
                const int c = active ? active[s + q] : s + q;
                if ((unsigned)c < (unsigned)d_out) b[q] = bias[c];
            }
        }
    }
    __device__ bool wants_stored() const { return z != nullptr; }
    template <int V> __device__ void stored(int m, int s, int valid, float (&v)[V]) {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] += b[q];
        store_values<T, V>(z + (size_t)m * n_active + s, v, valid);
    }
    template <int V> __device__ void gap_values(int gaps, float (&flat)[V]) const {
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (gaps >> q & 1) flat[q] = act_value(flat[q], act);
    }
    template <int V> __device__ void listed(int m, int c, int first, int valid, float (&v)[V], int gaps, const float (&flat)[V]) const {
        const size_t at = (size_t)m * d_out + c;
        float r[V] = {};
        if (residual) load_values<TY, V>(residual + at, r, valid, first);
#pragma unroll
        for (int q = 0; q < V; ++q) {
            v[q] = gaps >> q & 1 ? flat[q] : act_value(v[q], act);
            if (residual) v[q] += r[q];
        }
        store_values<TY, V>(y + at, v, valid, first);
    }
    // the ablated columns lo .. hi - 1
    __device__ void ablated(int m, int lo, int hi) {
        for (int c = max(lo, 0); c < min(hi, d_out); ++c) {
            const size_t at = (size_t)m * d_out + c;
            const float v = act_value(bias ? bias[c] : 0.0f, act);
            y[at] = from_float<TY>(residual ? v + to_float(residual[at]) : v);
        }
    }
    template <int V> __device__ void row(int m, int s, int valid, float (&v)[V]) {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] += b[q];
        if (z) store_values<T, V>(z + (size_t)m * n_active + s, v, valid);
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = act_value(v[q], act);
        if (!active) {
            const size_t at = (size_t)m * d_out + s;
            if (residual) {
                float r[V];
                load_values<TY, V>(residual + at, r, valid);
#pragma unroll
                for (int q = 0; q < V; ++q) v[q] += r[q];
            }
            store_values<TY, V>(y + at, v, valid);
            return;
        }
        // stored neuron s + q writes the ablated columns in front of it too, the last one those behind it
#pragma unroll
        for (int q = 0; q < V; ++q) {
            if (q >= valid) break;
            const int c = active[s + q];
            ablated(m, s + q > 0 ? active[s + q - 1] + 1 : 0, c);
            if ((unsigned)c < (unsigned)d_out) {
                const size_t at = (size_t)m * d_out + c;
                y[at] = from_float<TY>(residual ? v[q] + to_float(residual[at]) : v[q]);
            }
            if (s + q == n_active - 1) ablated(m, c + 1, d_out);
        }
    }
};

template <typename T>
struct GatedOut {
    static constexpr bool kListed = false;
    const float *bias_g, *bias_u;
    int n;
    T *h, *g, *u;   // g and u: nullptr where the caller does not keep them
    int act;
    float bg[8], bu[8];

    template <int V> __device__ void start(int c, int valid) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            bg[q] = bias_g && q < valid ? bias_g[c + q] : 0.0f;
            bu[q] = bias_u && q < valid ? bias_u[c + q] : 0.0f;
        }
    }
    template <int V> __device__ void row(int m, int c, int valid, float (&v)[V], float (&w)[V]) {
        const size_t at = (size_t)m * n + c;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            v[q] += bg[q];
            w[q] += bu[q];
        }
        if (g) {
            store_values<T, V>(g + at, v, valid);
            store_values<T, V>(u + at, w, valid);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = act_value(v[q], act) * w[q];
        store_values<T, V>(h + at, v, valid);
    }
};

// No stored neuron: every column is act(bias) plus the residual.
template <typename TY>
__global__ __launch_bounds__(256) void k_bias_rows(const float* __restrict__ bias, const TY* residual, int B, int d_out, TY* y, int act) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= d_out) return;
    const float v = act_value(bias ? bias[c] : 0.0f, act);
    for (int m = blockIdx.y; m < B; m += gridDim.y) {
        const size_t at = (size_t)m * d_out + c;
        y[at] = from_float<TY>(residual ? v + to_float(residual[at]) : v);
    }
}

static DensePlan plan_forward(int B, int d_in, int n, bool f32, bool pair) {
    return plan_dense(B, n, f32 ? stages_of<float>(d_in) : stages_of<uint16_t>(d_in), f32, pair, d_in % (f32 ? 4 : 8) == 0);
}

template <typename T, typename TY>
static srigl_status linear_act(const void* x, int B, int d_in, const void* Wd, const int32_t* active, int n, const float* bias, const void* residual, int d_out,
                               void* y, void* z, int act, void* ws, size_t ws_bytes, hipStream_t st) {
    const DensePlan plan = plan_forward(B, d_in, n, sizeof(T) == 4, false);
    const bool few = few_rows(B, d_in, sizeof(T) == 4, false);
    if (!few && !scratch_fits(ws, ws_bytes, part_bytes(plan, B, n, false))) return SRIGL_ERR_CAPACITY;
    if (n == 0) {
        hipLaunchKernelGGL(k_bias_rows<TY>, dim3((unsigned)((d_out + 255) / 256), (unsigned)std::min(B, 65535)), dim3(256), 0, st, bias, (const TY*)residual, B, d_out,
                           (TY*)y, act);
        return hip_ok(hipGetLastError());
    }
    const RowsOf<T> a{(const T*)x, d_in, B - 1, d_in}, w{(const T*)Wd, d_in, n - 1, d_in};
    const LinearOut<T, TY> out{n == d_out ? nullptr : active, n, bias, (const TY*)residual, d_out, (TY*)y, (T*)z, act, {}};
    if (few) return launch_few<T, false>((const T*)x, B, d_in, (const T*)Wd, 0, n, out, st);
    return launch_dense<T, false>(a, w, B, n, stages_of<T>(d_in), plan, out, (float*)ws, st);
}

template <typename T>
static srigl_status gated(const void* x, int B, int d_in, const void* Wg, const void* Wu, int n, const float* bias_g, const float* bias_u, int act, void* h, void* g,
                          void* u, void* ws, size_t ws_bytes, hipStream_t st) {
    const DensePlan plan = plan_forward(B, d_in, n, sizeof(T) == 4, true);
    const bool few = few_rows(B, d_in, sizeof(T) == 4, true);
    if (!few && !scratch_fits(ws, ws_bytes, part_bytes(plan, B, n, true))) return SRIGL_ERR_CAPACITY;
    const RowsOf<T> a{(const T*)x, d_in, B - 1, d_in};
    const PairedRows<T, 32> w{(const T*)Wg, bytes_between(Wg, Wu), d_in, n - 1, d_in};
    const GatedOut<T> out{bias_g, bias_u, n, (T*)h, (T*)g, (T*)u, act, {}, {}};
    if (few) return launch_few<T, true>((const T*)x, B, d_in, (const T*)Wg, bytes_between(Wg, Wu), n, out, st);
    return launch_dense<T, true>(a, w, B, n, stages_of<T>(d_in), plan, out, (float*)ws, st);
}

}  // namespace srigl

using namespace srigl;

extern "C" {

size_t srigl_structured_act_workspace_bytes(int32_t B, int32_t d_in, int32_t n_active, srigl_dtype dtype) {
    if (B < 0 || d_in < 0 || n_active < 0 || B > kMaxSide || d_in > kMaxSide || n_active > kMaxSide || !known_dtype(dtype)) return 0;
    return few_rows(B, d_in, dtype == SRIGL_F32, false) ? 0 : part_bytes(plan_forward(B, d_in, n_active, dtype == SRIGL_F32, false), B, n_active, false);
}

srigl_status srigl_structured_linear_fwd_act(const void* x, srigl_dtype x_dtype, int32_t B, int32_t d_in, const void* Wd, srigl_dtype w_dtype, const int32_t* active,
                                             int32_t n_active, const float* bias, const void* residual, int32_t d_out, void* y, srigl_dtype y_dtype, void* z,
                                             srigl_activation act, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || d_in < 0 || n_active < 0 || d_out < 0 || n_active > d_out) return SRIGL_ERR_INVALID_ARG;
    if (!known_dtype(x_dtype) || !known_dtype(w_dtype) || !known_dtype(y_dtype) || !known_act(act)) return SRIGL_ERR_INVALID_ARG;
    if (x_dtype != w_dtype || (y_dtype != x_dtype && y_dtype != SRIGL_F32)) return SRIGL_ERR_UNSUPPORTED;
    if (B > kMaxSide || d_in > kMaxSide || d_out > kMaxSide) return SRIGL_ERR_UNSUPPORTED;
    if (active == nullptr && n_active != d_out && n_active != 0) return SRIGL_ERR_INVALID_ARG;
    if (B == 0 || d_out == 0) return SRIGL_OK;
    if (y == nullptr || (n_active > 0 && d_in > 0 && (x == nullptr || Wd == nullptr))) return SRIGL_ERR_INVALID_ARG;
    if (astray(dtype_bytes(x_dtype), {x, Wd, z}) || astray(dtype_bytes(y_dtype), {y, residual}) || astray(4, {bias, active}) || astray(16, {workspace})) return SRIGL_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_dtype == SRIGL_F32) return linear_act<float, float>(x, B, d_in, Wd, active, n_active, bias, residual, d_out, y, z, act, workspace, workspace_bytes, st);
    if (y_dtype == SRIGL_F32) return linear_act<uint16_t, float>(x, B, d_in, Wd, active, n_active, bias, residual, d_out, y, z, act, workspace, workspace_bytes, st);
    return linear_act<uint16_t, uint16_t>(x, B, d_in, Wd, active, n_active, bias, residual, d_out, y, z, act, workspace, workspace_bytes, st);
}

size_t srigl_gated_workspace_bytes(int32_t B, int32_t d_in, int32_t n, srigl_dtype dtype) {
    if (B < 0 || d_in < 0 || n < 0 || B > kMaxSide || d_in > kMaxSide || n > kMaxSide || !known_dtype(dtype)) return 0;
    return few_rows(B, d_in, dtype == SRIGL_F32, true) ? 0 : part_bytes(plan_forward(B, d_in, n, dtype == SRIGL_F32, true), B, n, true);
}

srigl_status srigl_gated_linear_fwd(const void* x, srigl_dtype x_dtype, int32_t B, int32_t d_in, const void* Wg, const void* Wu, srigl_dtype w_dtype, int32_t n,
                                    const float* bias_g, const float* bias_u, srigl_activation act, void* h, void* g, void* u, void* workspace,
                                    size_t workspace_bytes, void* stream) {
    if (B < 0 || d_in < 0 || n < 0 || !known_dtype(x_dtype) || !known_dtype(w_dtype) || !known_act(act)) return SRIGL_ERR_INVALID_ARG;
    if (x_dtype != w_dtype || B > kMaxSide || d_in > kMaxSide || n > kMaxSide) return SRIGL_ERR_UNSUPPORTED;
    if ((g == nullptr) != (u == nullptr)) return SRIGL_ERR_INVALID_ARG;
    if (B == 0 || n == 0) return SRIGL_OK;
    if (h == nullptr || (d_in > 0 && (x == nullptr || Wg == nullptr || Wu == nullptr))) return SRIGL_ERR_INVALID_ARG;
    if (astray(dtype_bytes(x_dtype), {x, Wg, Wu, h, g, u}) || astray(4, {bias_g, bias_u}) || astray(16, {workspace})) return SRIGL_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_dtype == SRIGL_F32) return gated<float>(x, B, d_in, Wg, Wu, n, bias_g, bias_u, act, h, g, u, workspace, workspace_bytes, st);
    return gated<uint16_t>(x, B, d_in, Wg, Wu, n, bias_g, bias_u, act, h, g, u, workspace, workspace_bytes, st);
}

}  // extern "C"
