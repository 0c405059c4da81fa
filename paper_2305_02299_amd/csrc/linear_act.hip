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
// 145000 timings in graphs, every tile and 1 to 16 parts of 26000 random products (17 to 2048 rows, 100 to 4096 wide, 100 to 16384 neurons): 4 to 10 % a timing; the tile and parts of smallest time are 0.3
// to 2 % behind the fastest on average by kind and type, 9 % at worst in 95 of 100, 34 % at worst.  (fp32 was timed with the parts of values cut off in place of rounded, 0 to 7 % faster.)
struct DenseModel {
    int kind, f32, direct, tile, slots;
    float us[7];   // fixed, round, per_k, per_k_full, results, second, part
};
static const DenseModel kDenseModels[] = {
    {0, 0, 0, 0, 512, {4.47f, 1.49f, 6.49f, 4.98f, 0.904f, 2.48f, 1.67f}},
    {0, 0, 0, 1, 512, {10.8f, 0.0f, 12.6f, 9.99f, 0.63f, 1.49f, 1.5f}},
    {0, 0, 1, 0, 512, {3.45f, 2.42f, 2.78f, 4.74f, 0.441f, 2.52f, 2.29f}},
    {0, 0, 1, 1, 256, {4.08f, 2.88f, 5.65f, 4.3f, 0.355f, 3.02f, 1.66f}},
    {0, 0, 1, 2, 256, {6.23f, 2.42f, 8.37f, 5.95f, 0.473f, 3.16f, 1.48f}},
    {0, 0, 1, 3, 256, {7.88f, 4.07f, 15.1f, 10.5f, 0.285f, 3.67f, 1.16f}},
    {0, 0, 1, 4, 512, {3.38f, 2.13f, 3.06f, 5.78f, 0.207f, 2.82f, 1.73f}},
    {0, 0, 1, 5, 512, {6.44f, 0.0f, 5.73f, 14.0f, 0.331f, 3.25f, 1.49f}},
    {0, 1, 0, 0, 512, {5.57f, 0.363f, 19.8f, 13.9f, 1.26f, 2.37f, 1.98f}},
    {0, 1, 0, 1, 512, {10.9f, 0.0f, 49.0f, 32.5f, 0.884f, 0.751f, 1.53f}},
    {0, 1, 1, 0, 256, {6.46f, 0.0f, 15.3f, 0.0f, 1.42f, 2.9f, 1.86f}},
    {0, 1, 1, 1, 256, {7.6f, 4.37f, 31.1f, 10.6f, 1.09f, 2.11f, 1.65f}},
    {0, 1, 1, 2, 256, {10.3f, 2.36f, 56.2f, 17.2f, 0.719f, 3.11f, 1.49f}},
    {0, 1, 1, 4, 512, {4.87f, 0.696f, 17.7f, 14.6f, 1.06f, 3.08f, 2.12f}},
    {0, 1, 1, 5, 256, {11.3f, 0.0f, 35.1f, 7.87f, 0.607f, 2.8f, 1.23f}},
    {1, 0, 0, 0, 1024, {7.51f, 0.0f, 9.0f, 21.7f, 0.416f, 2.47f, 1.7f}},
    {1, 0, 0, 1, 512, {10.4f, 0.0f, 12.5f, 10.0f, 0.361f, 2.25f, 1.3f}},
    {1, 0, 1, 0, 256, {3.24f, 3.56f, 4.42f, 2.4f, 0.422f, 3.2f, 1.65f}},
    {1, 0, 1, 1, 256, {3.63f, 3.11f, 5.8f, 3.86f, 0.285f, 3.48f, 1.7f}},
    {1, 0, 1, 2, 256, {5.45f, 2.68f, 8.6f, 4.99f, 0.452f, 3.95f, 1.51f}},
    {1, 0, 1, 3, 256, {7.49f, 3.56f, 15.6f, 8.22f, 0.328f, 4.39f, 1.16f}},
    {1, 0, 1, 4, 1280, {4.34f, 1.72f, 4.83f, 25.8f, 0.394f, 3.38f, 1.86f}},
    {1, 0, 1, 5, 512, {6.0f, 0.0f, 6.05f, 13.1f, 0.359f, 4.03f, 1.5f}},
    {1, 1, 0, 0, 768, {6.89f, 0.0f, 29.4f, 44.4f, 0.719f, 3.07f, 1.73f}},
    {1, 1, 0, 1, 512, {9.19f, 0.0f, 48.5f, 36.9f, 0.664f, 2.69f, 1.42f}},
    {1, 1, 1, 0, 256, {3.59f, 3.85f, 22.5f, 6.51f, 0.74f, 3.73f, 1.73f}},
    {1, 1, 1, 1, 256, {6.02f, 4.16f, 31.8f, 10.1f, 0.89f, 3.78f, 1.76f}},
    {1, 1, 1, 2, 256, {7.95f, 2.77f, 56.8f, 17.0f, 0.724f, 5.03f, 1.52f}},
    {1, 1, 1, 4, 1280, {5.49f, 0.747f, 24.5f, 81.3f, 0.973f, 3.91f, 1.97f}},
    {1, 1, 1, 5, 256, {9.44f, 0.0f, 37.4f, 5.78f, 0.584f, 4.65f, 1.25f}},
    {2, 0, 0, 0, 1536, {5.67f, 0.0f, 11.0f, 13.7f, 0.375f, 2.93f, 2.48f}},
    {2, 0, 0, 1, 1536, {8.5f, 0.0f, 16.4f, 30.0f, 0.123f, 3.27f, 1.67f}},
    {2, 0, 1, 0, 256, {7.24f, 0.111f, 3.43f, 1.18f, 0.444f, 2.95f, 2.83f}},
    {2, 0, 1, 1, 256, {7.74f, 1.77f, 5.71f, 3.68f, 0.271f, 3.56f, 2.31f}},
    {2, 0, 1, 2, 256, {9.01f, 0.524f, 8.63f, 5.41f, 0.424f, 4.03f, 1.84f}},
    {2, 0, 1, 3, 256, {10.2f, 1.13f, 15.7f, 9.17f, 0.573f, 5.14f, 1.41f}},
    {2, 0, 1, 4, 1024, {6.36f, 0.0f, 5.98f, 8.31f, 0.525f, 3.16f, 2.84f}},
    {2, 0, 1, 5, 1280, {8.36f, 0.0f, 8.42f, 29.2f, 0.0758f, 3.71f, 1.83f}},
    {2, 1, 0, 0, 1536, {2.33f, 3.37f, 29.8f, 48.8f, 0.708f, 3.16f, 2.76f}},
    {2, 1, 0, 1, 512, {8.58f, 0.0f, 62.7f, 29.3f, 0.431f, 3.62f, 1.74f}},
    {2, 1, 1, 0, 512, {5.81f, 1.15f, 16.0f, 15.3f, 0.717f, 3.14f, 2.9f}},
    {2, 1, 1, 1, 256, {8.79f, 2.53f, 33.5f, 11.5f, 0.58f, 3.8f, 2.19f}},
    {2, 1, 1, 2, 256, {11.6f, 0.829f, 59.2f, 19.5f, 0.17f, 4.56f, 1.87f}},
    {2, 1, 1, 4, 1280, {1.72f, 3.86f, 20.5f, 45.8f, 0.701f, 3.66f, 2.73f}},
    {2, 1, 1, 5, 512, {9.81f, 0.0f, 38.3f, 40.2f, 0.277f, 4.27f, 1.78f}},
    {3, 0, 0, 0, 1536, {6.62f, 0.0f, 9.87f, 18.1f, 0.397f, 2.33f, 2.54f}},
    {3, 0, 0, 1, 768, {9.12f, 0.0f, 16.4f, 19.7f, 0.362f, 3.69f, 1.4f}},
    {3, 0, 1, 0, 512, {5.54f, 1.42f, 3.67f, 6.03f, 0.456f, 2.82f, 3.01f}},
    {3, 0, 1, 1, 256, {5.95f, 3.02f, 7.29f, 4.57f, 0.351f, 4.44f, 1.73f}},
    {3, 0, 1, 2, 256, {7.17f, 1.86f, 10.3f, 8.14f, 0.376f, 4.97f, 1.41f}},
    {3, 0, 1, 3, 256, {7.87f, 3.66f, 17.0f, 13.5f, 0.238f, 6.26f, 1.08f}},
    {3, 0, 1, 4, 1024, {6.48f, 0.107f, 5.4f, 12.0f, 0.53f, 2.77f, 2.67f}},
    {3, 0, 1, 5, 512, {7.98f, 0.517f, 8.49f, 11.6f, 0.434f, 4.84f, 1.38f}},
    {3, 1, 0, 0, 1536, {6.03f, 0.0f, 30.0f, 69.5f, 0.569f, 2.96f, 2.23f}},
    {3, 1, 0, 1, 512, {9.02f, 0.0f, 60.8f, 41.9f, 0.6f, 4.1f, 1.36f}},
    {3, 1, 1, 0, 512, {5.76f, 0.733f, 17.2f, 16.6f, 1.22f, 3.5f, 2.66f}},
    {3, 1, 1, 1, 256, {6.45f, 4.21f, 36.6f, 13.2f, 0.673f, 4.81f, 1.57f}},
    {3, 1, 1, 2, 256, {8.13f, 3.59f, 63.4f, 22.2f, 0.607f, 6.19f, 1.24f}},
    {3, 1, 1, 4, 1280, {6.26f, 0.0f, 18.0f, 55.0f, 0.95f, 3.2f, 2.51f}},
    {3, 1, 1, 5, 512, {10.1f, 0.0f, 37.8f, 44.6f, 0.846f, 5.05f, 1.42f}},
};

// one product of a model's kind
struct DenseShape {
    const DenseModel& m;
    double k, sums;
    long long tiles, padded;
    int stages;
    DenseShape(const DenseModel& model, int M, int N, int stages_) : m(model), stages(stages_) {
        static const int kRows[] = {64, 128, 256, 256, 64, 128}, kCols[] = {64, 128, 128, 256, 64, 128}, kPairCols[] = {64, 64, 64, 128, 64, 64};
        const bool pair = m.kind == kDensePair;
        const long long bm = kRows[m.tile], bn = (pair ? kPairCols : kCols)[m.tile];
        tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), padded = (tiles + kXcds - 1) / kXcds * kXcds;
        k = 1e-3 * stages * (m.f32 ? 32 : 64), sums = 1e-6 * M * N * (pair ? 2 : 1);
    }
    // two stages to a part, parts side by side
    bool allowed(int parts) const { return parts == 1 || (parts * 2 <= stages && tiles * parts <= (m.direct && m.tile < kTileS2 ? 560 : 1200)); }
    double groups(int parts) const { return (double)(parts > 1 ? padded * parts : tiles); }
    double us(int parts) const {
        const double g = groups(parts);
        return m.us[0] + std::ceil(g / m.slots) * (m.us[1] + m.us[2] * k / parts) + g / m.slots * m.us[3] * k / parts + m.us[4] * sums + (parts > 1 ? m.us[5] + m.us[6] * parts * sums : 0.0);
    }
};

static DensePlan fastest(DenseKind kind, int M, int N, int stages, bool f32, bool direct, int tile, double* best_us) {
    DensePlan best{kTileS, 1};
    *best_us = 0.0;
    for (const DenseModel& m : kDenseModels) {
        if (m.kind != (int)kind || m.f32 != f32 || m.direct != direct || (tile >= 0 && m.tile != tile)) continue;
        const DenseShape shape(m, M, N, stages);
        for (int parts = 1; parts <= 16 && shape.allowed(parts); ++parts) {
            const double us = shape.us(parts);
            if (*best_us == 0.0 || us < *best_us) best = {m.tile, parts}, *best_us = us;
        }
    }
    return best;
}

DensePlan plan_dense(DenseKind kind, int M, int N, int stages, bool f32, bool direct) {
    if (M <= 0 || N <= 0) return {kTileS, 1};
    struct Key { int32_t M, N, stages, form; };
    static thread_local DecisionCache<Key, DensePlan, 64> cache;
    return cache.get(Key{M, N, stages, f32 + 2 * direct + 4 * (int)kind}, [&] {
        double us;
        return fastest(kind, M, N, stages, f32, direct, -1, &us);
    });
}

// Two products in one launch, fitted likewise to 68000 timings of 5400 pairs: fixed, a round; by 1000 elements of K a round of the mean workgroup, the work of all of them and the longest one; results; second, part.
struct DenseTwoModel {
    int f32, direct, tile, slots;
    float us[8];
};
static const DenseTwoModel kDenseTwoModels[] = {
    {0, 0, 0, 512, {5.3f, 0.413f, 0.528f, 4.79f, 10.6f, 0.0f, 3.59f, 2.04f}},
    {0, 0, 1, 1024, {7.29f, 1.09f, 1.8f, 22.2f, 15.5f, 0.0f, 4.11f, 1.47f}},
    {0, 1, 0, 512, {6.25f, 1.3f, 0.81f, 6.6f, 2.67f, 0.0373f, 2.68f, 2.79f}},
    {0, 1, 1, 256, {7.64f, 2.16f, 2.02f, 5.71f, 4.46f, 0.03f, 3.58f, 1.84f}},
    {0, 1, 2, 256, {8.07f, 1.54f, 3.16f, 8.15f, 7.46f, 0.0f, 4.11f, 1.48f}},
    {0, 1, 3, 256, {8.59f, 3.05f, 2.66f, 12.7f, 14.4f, 0.0f, 5.01f, 1.2f}},
    {0, 1, 4, 256, {6.16f, 0.372f, 1.0f, 1.82f, 5.31f, 0.0f, 3.25f, 1.92f}},
    {0, 1, 5, 256, {7.69f, 0.862f, 0.194f, 6.22f, 7.86f, 0.0f, 4.22f, 1.29f}},
    {1, 0, 0, 512, {5.35f, 0.302f, 0.933f, 18.3f, 29.0f, 0.0f, 3.26f, 2.43f}},
    {1, 0, 1, 512, {5.78f, 2.25f, 6.13f, 41.6f, 59.0f, 0.0f, 3.81f, 1.62f}},
    {1, 1, 0, 256, {6.62f, 0.89f, 2.96f, 7.06f, 14.1f, 0.0f, 2.61f, 2.59f}},
    {1, 1, 1, 256, {8.29f, 3.76f, 5.81f, 20.0f, 28.6f, 0.0f, 3.28f, 1.71f}},
    {1, 1, 2, 256, {8.06f, 4.46f, 9.22f, 27.1f, 53.3f, 0.0f, 4.42f, 1.4f}},
    {1, 1, 4, 256, {5.4f, 0.784f, 0.0f, 9.1f, 19.5f, 0.0f, 3.43f, 1.63f}},
    {1, 1, 5, 256, {8.91f, 1.72f, 0.17f, 24.4f, 36.1f, 0.0611f, 4.05f, 1.19f}},
};

// One launch where it is expected to be ahead of two: on 9 of 10 of those pairs, by 20 % of both products on average (1 to 3 % behind the best tile and parts).
DensePlans plan_gradients(int B, int d_in, int K_stages, int rows, int B_stages, bool f32, bool direct) {
    struct Key { int32_t B, d_in, K_stages, rows, B_stages, form; };
    static thread_local DecisionCache<Key, DensePlans, 64> cache;
    if (B <= 0 || d_in <= 0 || rows <= 0) return {{kTileS, 1}, {kTileS, 1}, false};
    return cache.get(Key{B, d_in, K_stages, rows, B_stages, f32 + 2 * direct}, [&] {
        DensePlans best{};
        double us_x, us_W;
        best.dx = fastest(kDenseGradX, B, d_in, K_stages, f32, direct, -1, &us_x);
        best.dW = fastest(kDenseGradW, rows, d_in, B_stages, f32, direct, -1, &us_W);
        double best_us = us_x + us_W;
        if (best_us > 250.0) return best;   // (beyond what was fitted; each in its own tile is ahead by 2 %: bf16 4096 x 16384 at 2048 rows)
        for (const DenseTwoModel& m : kDenseTwoModels) {
            if (m.f32 != f32 || m.direct != direct) continue;
            const DenseModel shape_of{kDenseGradX, f32, direct, m.tile, m.slots, {}};
            const DenseShape x(shape_of, B, d_in, K_stages), W(shape_of, rows, d_in, B_stages);
            for (int a = 1; a <= 16 && x.allowed(a); ++a)
                for (int b = 1; b <= 16 && W.allowed(b); ++b) {
                    const double gx = (double)x.padded * a, gW = (double)W.padded * b, work = gx * x.k / a + gW * W.k / b;
                    const double us = m.us[0] + std::ceil((gx + gW) / m.slots) * (m.us[1] + m.us[2] * work / (gx + gW)) + m.us[3] * work / m.slots + m.us[4] * std::max(x.k / a, W.k / b) +
                                      m.us[5] * (x.sums + W.sums) + (a > 1 || b > 1 ? m.us[6] : 0.0) + m.us[7] * ((a > 1 ? a * x.sums : 0.0) + (b > 1 ? b * W.sums : 0.0));
                    if (us < best_us) best = {{m.tile, a}, {m.tile, b}, true}, best_us = us;
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
        act_values<V>(v, act);
#pragma unroll
        for (int q = 0; q < V; ++q) {
            v[q] = gaps >> q & 1 ? flat[q] : v[q];
            if (residual) v[q] += r[q];
        }
        store_values<TY, V>(y + at, v, valid, first);
    }
    __device__ float ablated_value(int c) const { return act_value(bias ? bias[c] : 0.0f, act); }
    // rows m0 .. m1 - 1, ROWS at most, of an ablated column; the residual's values are requested together
    template <int ROWS> __device__ void ablated_rows(int c, int m0, int m1, float flat) const {
        TY r[ROWS] = {};
        if (residual)
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (m0 + k < m1) r[k] = residual[(size_t)(m0 + k) * d_out + c];
#pragma unroll
        for (int k = 0; k < ROWS; ++k)
            if (m0 + k < m1) y[(size_t)(m0 + k) * d_out + c] = from_float<TY>(residual ? flat + to_float(r[k]) : flat);
    }
    template <int V> __device__ void row(int m, int s, int valid, float (&v)[V]) {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] += b[q];
        if (z) store_values<T, V>(z + (size_t)m * n_active + s, v, valid);
        act_values<V>(v, act);
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
#pragma unroll
        for (int q = 0; q < V; ++q) {
            if (q >= valid) break;
            const int c = active[s + q];
            if ((unsigned)c < (unsigned)d_out) {
                const size_t at = (size_t)m * d_out + c;
                y[at] = from_float<TY>(residual ? v[q] + to_float(residual[at]) : v[q]);
            }
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
        act_values<V>(v, act);
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] *= w[q];
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
    return launch_dense<T, false>(DenseProduct<RowsOf<T>, RowsOf<T>, LinearOut<T, TY>>{a, w, out, B, n, stages_of<T>(d_in), plan.parts, (float*)ws}, plan.tile, st);
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
    return launch_dense<T, true>(DenseProduct<RowsOf<T>, PairedRows<T, 32>, GatedOut<T>>{a, w, out, B, n, stages_of<T>(d_in), plan.parts, (float*)ws}, plan.tile, st);
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
