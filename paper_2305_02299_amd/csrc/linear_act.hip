// One layer in the structured-only form with bias, activation and residual behind the product, and a gated block (gfx950):
//     z[b][s] = bias[a(s)] + sum_j Wd[s][j] x[b][j],   y[b][a(s)] = act(z[b][s]) + r[b][a(s)],   other columns c: act(bias[c]) + r[b][c]
//     h[b][c] = act(bg[c] + sum_j Wg[c][j] x[b][j]) * (bu[c] + sum_j Wu[c][j] x[b][j])
// The gated block is one product over both weight matrices' rows: a workgroup's tile holds the same rows of both, each wavefront the gate's sums and the
// up-projection's of the same neurons, so that they meet in the epilogue and neither projection goes to memory (unless the caller keeps them for
// the backward pass).
#include "dense_tile.h"

namespace srigl {

// Expected time (us) of a product in a tile and `parts` parts of K: a fixed part, a part a round of workgroups over the compute units and, by 1000 elements of K, a part a round and one that follows how
// full the rounds are, a part per million results, a second launch and the parts' sums (a million of them written and read) where there are several.  Non-negative least squares on the relative error of
// 170000 timings in graphs, every tile and 1 to 16 parts of 29000 random products (17 to 2048 rows, 100 to 4096 wide, 100 to 16384 neurons): 3 to 12 % a timing; the tile and parts of smallest time are 0.1
// to 1.1 % behind the fastest on average by kind and type, 8 % at worst in 95 of 100, 37 % at worst.
struct DenseModel {
    int kind, f32, direct, tile, slots;
    float us[7];   // fixed, round, per_k, per_k_full, results, second, part
};
static const DenseModel kDenseModels[] = {
    {0, 0, 0, 0, 512, {4.47f, 1.49f, 6.49f, 4.98f, 0.904f, 2.48f, 1.67f}},
    {0, 0, 0, 1, 512, {10.8f, 0.0f, 12.6f, 9.99f, 0.63f, 1.49f, 1.5f}},
    {0, 0, 1, 0, 512, {3.49f, 2.7f, 2.91f, 4.71f, 0.509f, 2.0f, 2.48f}},
    {0, 0, 1, 1, 256, {4.8f, 3.06f, 5.67f, 4.17f, 0.502f, 2.24f, 1.63f}},
    {0, 0, 1, 2, 256, {7.47f, 2.08f, 8.42f, 5.26f, 0.699f, 2.13f, 1.48f}},
    {0, 0, 1, 3, 256, {10.5f, 3.56f, 15.1f, 9.99f, 0.505f, 1.13f, 1.14f}},
    {0, 1, 0, 0, 256, {5.67f, 0.0315f, 20.9f, 0.0f, 1.11f, 2.17f, 1.88f}},
    {0, 1, 0, 1, 256, {10.2f, 0.0f, 66.2f, 2.89f, 0.684f, 0.902f, 1.5f}},
    {0, 1, 1, 0, 256, {5.59f, 0.409f, 16.9f, 1.5f, 1.22f, 2.63f, 1.91f}},
    {0, 1, 1, 1, 256, {6.32f, 2.1f, 56.7f, 7.6f, 0.948f, 3.35f, 1.7f}},
    {1, 0, 0, 0, 1024, {7.51f, 0.0f, 9.0f, 21.7f, 0.416f, 2.47f, 1.7f}},
    {1, 0, 0, 1, 512, {10.4f, 0.0f, 12.5f, 10.0f, 0.361f, 2.25f, 1.3f}},
    {1, 0, 1, 0, 256, {3.6f, 3.77f, 4.39f, 2.74f, 0.488f, 2.62f, 1.53f}},
    {1, 0, 1, 1, 256, {4.13f, 3.35f, 5.59f, 4.26f, 0.343f, 2.83f, 1.63f}},
    {1, 0, 1, 2, 256, {6.5f, 2.58f, 8.5f, 4.94f, 0.55f, 2.73f, 1.46f}},
    {1, 0, 1, 3, 256, {9.16f, 3.71f, 15.3f, 9.14f, 0.348f, 2.44f, 1.12f}},
    {1, 1, 0, 0, 256, {6.75f, 0.0f, 36.2f, 0.0f, 0.531f, 2.66f, 1.51f}},
    {1, 1, 0, 1, 256, {8.73f, 0.0f, 65.8f, 0.0f, 0.653f, 2.51f, 1.38f}},
    {1, 1, 1, 0, 256, {3.88f, 3.3f, 31.4f, 5.3f, 0.807f, 3.44f, 1.57f}},
    {1, 1, 1, 1, 256, {5.21f, 2.3f, 57.0f, 6.95f, 0.709f, 4.32f, 1.76f}},
    {2, 0, 0, 0, 1536, {5.67f, 0.0f, 11.0f, 13.7f, 0.375f, 2.93f, 2.48f}},
    {2, 0, 0, 1, 1536, {8.5f, 0.0f, 16.4f, 30.0f, 0.123f, 3.27f, 1.67f}},
    {2, 0, 1, 0, 256, {7.2f, 0.119f, 3.6f, 1.06f, 0.503f, 2.87f, 2.85f}},
    {2, 0, 1, 1, 256, {7.95f, 1.58f, 5.67f, 3.77f, 0.394f, 3.38f, 2.38f}},
    {2, 0, 1, 2, 256, {9.2f, 0.299f, 8.67f, 4.92f, 0.479f, 3.87f, 1.88f}},
    {2, 0, 1, 3, 256, {10.8f, 0.656f, 15.9f, 8.48f, 0.602f, 4.97f, 1.46f}},
    {2, 1, 0, 0, 1536, {1.59f, 3.58f, 28.0f, 67.0f, 1.34f, 2.57f, 2.99f}},
    {2, 1, 0, 1, 256, {7.69f, 0.0f, 76.2f, 0.0f, 0.777f, 4.15f, 1.17f}},
    {2, 1, 1, 0, 256, {6.79f, 0.0f, 17.0f, 1.88f, 0.676f, 2.97f, 2.47f}},
    {2, 1, 1, 1, 256, {8.5f, 0.0f, 57.7f, 8.49f, 0.138f, 4.35f, 2.22f}},
    {3, 0, 0, 0, 1536, {6.62f, 0.0f, 9.87f, 18.1f, 0.397f, 2.33f, 2.54f}},
    {3, 0, 0, 1, 768, {9.12f, 0.0f, 16.4f, 19.7f, 0.362f, 3.69f, 1.4f}},
    {3, 0, 1, 0, 512, {5.56f, 1.34f, 3.94f, 5.76f, 0.476f, 2.8f, 2.89f}},
    {3, 0, 1, 1, 256, {5.9f, 2.99f, 7.42f, 3.96f, 0.336f, 4.43f, 1.74f}},
    {3, 0, 1, 2, 256, {7.05f, 1.96f, 10.5f, 7.67f, 0.35f, 5.19f, 1.39f}},
    {3, 0, 1, 3, 256, {8.06f, 3.53f, 17.1f, 13.5f, 0.227f, 6.23f, 1.06f}},
    {3, 1, 0, 0, 1536, {5.45f, 0.0f, 26.5f, 99.4f, 0.553f, 2.66f, 2.28f}},
    {3, 1, 0, 1, 256, {8.31f, 0.0f, 75.8f, 1.78f, 0.473f, 4.59f, 1.09f}},
    {3, 1, 1, 0, 256, {5.74f, 0.608f, 17.4f, 3.12f, 0.575f, 2.99f, 2.14f}},
    {3, 1, 1, 1, 256, {6.12f, 1.75f, 58.2f, 13.0f, 0.623f, 5.07f, 1.69f}},
};

DensePlan plan_dense(DenseKind kind, int M, int N, int stages, bool f32, bool direct) {
    if (M <= 0 || N <= 0) return {kTileS, 1};
    struct Key { int32_t M, N, stages, form; };
    static thread_local DecisionCache<Key, DensePlan, 64> cache;
    return cache.get(Key{M, N, stages, f32 + 2 * direct + 4 * (int)kind}, [&] {
        DensePlan best{kTileS, 1};
        double best_us = 0.0;
        const bool pair = kind == kDensePair;
        const double k = 1e-3 * stages * (f32 ? 32 : 64), sums = 1e-6 * M * N * (pair ? 2 : 1);
        for (const DenseModel& m : kDenseModels) {
            if (m.kind != (int)kind || m.f32 != f32 || m.direct != direct) continue;
            static const int kRows[] = {64, 128, 256, 256}, kCols[] = {64, 128, 128, 256}, kPairCols[] = {64, 64, 64, 128};
            const long long bm = kRows[m.tile], bn = (pair ? kPairCols : kCols)[m.tile];
            const long long tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), padded = (tiles + kXcds - 1) / kXcds * kXcds;
            for (int parts = 1; parts <= 16; ++parts) {
                if (parts > 1 && (parts * 2 > stages || tiles * parts > (direct ? 560 : 1200))) break;   // two stages to a part, parts side by side
                const double groups = (double)(parts > 1 ? padded * parts : tiles), rounds = std::ceil(groups / m.slots);
                const double us = m.us[0] + rounds * (m.us[1] + m.us[2] * k / parts) + groups / m.slots * m.us[3] * k / parts + m.us[4] * sums +
                                  (parts > 1 ? m.us[5] + m.us[6] * parts * sums : 0.0);
                if (best_us == 0.0 || us < best_us) best = {m.tile, parts}, best_us = us;
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
    return plan_dense(pair ? kDensePair : kDenseForward, B, n, f32 ? stages_of<float>(d_in) : stages_of<uint16_t>(d_in), f32, d_in % (f32 ? 4 : 8) == 0);
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
