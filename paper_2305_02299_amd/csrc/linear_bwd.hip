// Gradients of a layer in the structured-only form and of a gated block (gfx950).
//     layer:  dz[b][s] = dy[b][a(s)] act'(z[b][s]);  dx = dz Wd;  dWd = dz^T x;  dbias[a(s)] = sum_b dz[b][s], of ablated columns c: act'(bias[c]) sum_b dy[b][c]
//     gated:  dg = dh u act'(g), du = dh act(g);  dx = dg Wg + du Wu;  dWg = dg^T x, dWu = du^T x;  dbias_g = sum_b dg, dbias_u = sum_b du
// One pass over the incoming gradient writes dz (dg | du) in the storage type to the workspace and the bias gradients' partial sums, from the values before that rounding; then
// come the two products.  The matrix units take bf16 values, so in bf16 dz is rounded once on its way into them; all sums run in fp32.  (dx and dW are then 0.0023 off the formula's in 2-norm, where their own rounding
// is 0.0017: a second bf16 part of dz would take that away for twice the multiplications, which are four fifths of a large call's time.)
// dz stands in the workspace with its rows padded by zeros to whole stages of K: the gated block's dg and du lie side by side, so that dx is one
// product over both matrices' lines and the weight gradients are one product too.
#include "dense_tile.h"
#include <type_traits>

namespace srigl {

constexpr int kPadK = 64;   // columns dz is padded to: whole stages of either type
static long long padded(int n) { return ((long long)n + kPadK - 1) / kPadK * kPadK; }

// first place in the ascending list whose entry is >= c
__device__ __forceinline__ int place_of(const int32_t* active, int n_active, int c) {
    int lo = 0, hi = n_active;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (active[mid] < c) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// One pass over the rows of the incoming gradient.  A workgroup takes 32 groups of V = 16 / sizeof(T) consecutive columns and a chunk of rows, eight rows side by side; the column sums of
// its eight row lanes meet in the LDS, and a chunk leaves one sum a column (no atomics: the order is fixed).  Bound by memory: three reads and two writes of 16 bytes a thread and row in the gated form;
// one column a thread and 2-byte accesses took 229 us on 2048 x 16384 bf16.
constexpr int kDzCols = 32, kDzRows = 8;

template <int V>
__device__ __forceinline__ void sum_row_lanes(float (*held)[kDzCols * V], float (&v)[V]) {
    const int cg = threadIdx.x % kDzCols, rl = threadIdx.x / kDzCols;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < V; ++q) held[rl][q * kDzCols + cg] = v[q];
    __syncthreads();
    if (rl == 0)
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int r = 1; r < kDzRows; ++r) v[q] += held[r][q * kDzCols + cg];
}

// dz[B][pitch] (pitch: n padded with zeros) and, per chunk of rows, its column sums in sums[chunk][n].  dz or sums: nullptr where not wanted.
template <typename T, typename TY>
__global__ __launch_bounds__(256) void k_dz_linear(const TY* __restrict__ dy, const T* __restrict__ z, int n, int B, int act, T* __restrict__ dz, int pitch,
                                                  float* __restrict__ sums, int rows) {
    constexpr int V = kPiece<T>;
    __shared__ float held[kDzRows][kDzCols * V];
    const int s = (int)((blockIdx.x * (unsigned)kDzCols + threadIdx.x % kDzCols) * V), m0 = blockIdx.y * rows, m1 = min(m0 + rows, B), valid = n - s;
    float sum[V] = {};
    if (s < pitch)
        for (int m = m0 + threadIdx.x / kDzCols; m < m1; m += kDzRows) {
            float v[V] = {}, zv[V] = {};
            if (valid > 0) {
                load_values<TY, V>(dy + (size_t)m * n + s, v, valid);
                if (act != SRIGL_ACT_NONE) {
                    float slope[V];
                    load_values<T, V>(z + (size_t)m * n + s, zv, valid);
                    act_slopes<V>(zv, slope, act);
#pragma unroll
                    for (int q = 0; q < V; ++q) v[q] = q < valid ? v[q] * slope[q] : 0.0f;
                }
            }
#pragma unroll
            for (int q = 0; q < V; ++q) sum[q] += v[q];
            if (dz) store_values<T, V>(dz + (size_t)m * pitch + s, v, V);
        }
    if (!sums) return;
    sum_row_lanes<V>(held, sum);
    if (threadIdx.x / kDzCols == 0 && valid > 0) store_values<float, V>(sums + (size_t)blockIdx.y * n + s, sum, valid);
}

// The same for a layer with ablated neurons.  A workgroup's columns of dy are those from behind the neuron in front of its own to its last one (the last workgroup's: to the end).  Where they fit, a row of
// them passes through the LDS, out of which a thread picks its V neurons' values, and all columns' sums are taken on the way; else the values are picked out of memory and the ablated columns' sums
// taken by a pass of their own.  Ablated columns go into sums[chunk][d_out] as they are.  (13108 of 16384 neurons, 2048 rows, bf16: 76 us; all picked out of memory and the ablated columns read again by
// a launch of their own 94; windows of columns, whose first and last neurons share a piece of dz with the windows beside, 107.)
template <typename T, typename TY>
__global__ __launch_bounds__(256) void k_dz_listed(const TY* __restrict__ dy, const T* __restrict__ z, const int32_t* __restrict__ active, int n, int B, int d_out, int act,
                                                  T* __restrict__ dz, int pitch, float* __restrict__ sums, int rows) {
    constexpr int V = kPiece<T>, OWN = kDzCols * V, PIECES = 2 * kDzCols, ROOM = PIECES * V;
    __shared__ float row[2][kDzRows][ROOM + 32], held[kDzRows][OWN];   // (column k of a row at k % V * PIECES + k / V; rows by turns half of the banks apart)
    __shared__ int stored[ROOM];
    const int cg = threadIdx.x % kDzCols, rl = threadIdx.x / kDzCols, m0 = blockIdx.y * rows, m1 = min(m0 + rows, B);
    const int s_first = blockIdx.x * OWN, s_behind = min(s_first + OWN, n), s = s_first + cg * V, valid = n - s;
    const int lo = s_first > 0 && s_first <= n ? max(active[s_first - 1] + 1, 0) : 0, hi = s_behind == n ? d_out : min(active[s_behind - 1] + 1, d_out), c0 = lo / V * V;
    const bool through = hi - c0 <= ROOM;
    int col[V], place[V];   // which columns the thread's neurons are, and where in the LDS they stand
    for (int k = threadIdx.x; k < ROOM; k += 256) stored[k] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < V; ++q) {
        col[q] = q < valid ? active[s + q] : -1;
        if (col[q] < lo || col[q] >= hi) col[q] = -1;
        const int k = col[q] - c0;
        place[q] = through && col[q] >= 0 ? k % V * PIECES + k / V : 0;
        if (through && col[q] >= 0) stored[k] = 1;
    }
    float sum[V] = {}, passed[2][V] = {};
    int buffer = 0;
    for (int base = m0; base < m1; base += kDzRows, buffer ^= 1) {
        const int m = base + rl;
        const bool there = m < m1;
        float v[V] = {}, zv[V] = {}, slope[V];
        if (there && valid > 0 && act != SRIGL_ACT_NONE) load_values<T, V>(z + (size_t)m * n + s, zv, valid);
        if (through) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int c = c0 + (j * kDzCols + cg) * V;
                float w[V] = {};
                if (there && c < hi) load_values<TY, V>(dy + (size_t)m * d_out + c, w, d_out - c);
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    passed[j][q] += w[q];
                    row[buffer][rl][q * PIECES + j * kDzCols + cg + (rl & 1) * 32] = w[q];
                }
            }
            __syncthreads();   // (the other buffer is written next: one barrier a row)
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = row[buffer][rl][place[q] + (rl & 1) * 32];
        } else if (there) {
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = to_float(dy[(size_t)m * d_out + max(col[q], 0)]);
        }
        if (!there || s >= pitch) continue;
        act_slopes<V>(zv, slope, act);
#pragma unroll
        for (int q = 0; q < V; ++q) {
            v[q] = col[q] >= 0 ? v[q] * slope[q] : 0.0f;
            sum[q] += v[q];
        }
        if (dz) store_values<T, V>(dz + (size_t)m * pitch + s, v, V);
    }
    if (!sums) return;
    float* const to = sums + (size_t)blockIdx.y * d_out;
    sum_row_lanes<V>(held, sum);
    if (rl == 0)
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (col[q] >= 0) to[col[q]] = sum[q];
    if (through) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sum_row_lanes<V>(held, passed[j]);
            if (rl == 0)
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    const int k = (j * kDzCols + cg) * V + q;
                    if (c0 + k >= lo && c0 + k < hi && !stored[k]) to[c0 + k] = passed[j][q];
                }
        }
    } else {
        for (int c = lo + (int)threadIdx.x; c < hi; c += 256) {
            const int at = n ? place_of(active, n, c) : 0;
            if (at < n && active[at] == c) continue;
            float v = 0.0f;
#pragma unroll 8
            for (int m = m0; m < m1; ++m) v += to_float(dy[(size_t)m * d_out + c]);
            to[c] = v;
        }
    }
}

// (dg | du)[B][2 pitch] and the column sums of both in sums[chunk][2 n]
template <typename T>
__global__ __launch_bounds__(256) void k_dz_gated(const T* __restrict__ dh, const T* __restrict__ g, const T* __restrict__ u, int n, int B, int act, T* __restrict__ dz,
                                                 int pitch, float* __restrict__ sums, int rows) {
    constexpr int V = kPiece<T>;
    __shared__ float held[kDzRows][kDzCols * V];
    const int c = (int)((blockIdx.x * (unsigned)kDzCols + threadIdx.x % kDzCols) * V), m0 = blockIdx.y * rows, m1 = min(m0 + rows, B), valid = n - c;
    float sg[V] = {}, su[V] = {};
    if (c < pitch)
        for (int base = m0 + threadIdx.x / kDzCols; base < m1; base += 2 * kDzRows) {   // (two rows' loads together)
            float d[2][V] = {}, gv[2][V] = {}, uv[2][V] = {}, slope[V];
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (valid > 0 && base + r * kDzRows < m1) {
                    const size_t at = (size_t)(base + r * kDzRows) * n + c;
                    load_values<T, V>(dh + at, d[r], valid);
                    load_values<T, V>(g + at, gv[r], valid);
                    load_values<T, V>(u + at, uv[r], valid);
                }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (base + r * kDzRows >= m1) break;
                act_slopes<V>(gv[r], slope, act);
                act_values<V>(gv[r], act);
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    const float dg = d[r][q] * uv[r][q] * slope[q], du = d[r][q] * gv[r][q];
                    sg[q] += gv[r][q] = q < valid ? dg : 0.0f;
                    su[q] += uv[r][q] = q < valid ? du : 0.0f;
                }
                T* const to = dz + (size_t)(base + r * kDzRows) * 2 * pitch + c;
                store_values<T, V>(to, gv[r], V);
                store_values<T, V>(to + pitch, uv[r], V);
            }
        }
    if (!sums) return;
    sum_row_lanes<V>(held, sg);
    sum_row_lanes<V>(held, su);
    if (threadIdx.x / kDzCols == 0 && valid > 0) {
        float* const to = sums + (size_t)blockIdx.y * 2 * n + c;
        store_values<float, V>(to, sg, valid);
        store_values<float, V>(to + n, su, valid);
    }
}

// Bias gradients from the chunks' sums, 64 columns to a workgroup, whose wavefronts take chunks by turns.  Columns [0, n) to first, [n, 2 n) to second (a layer: all to first, ablated
// columns times the slope at their bias).
struct SumChunks {
    const float* sums;
    int chunks, cols, n;
    const int32_t* active;
    int n_active;
    const float* bias;
    int act;
    float *first, *second;
    long long groups() const { return first || second ? (cols + 63ll) / 64 : 0; }
    __device__ __forceinline__ void operator()(unsigned char* smem, int group) const {
        float(*const held)[64] = reinterpret_cast<float(*)[64]>(smem);
        const int c = group * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        float v = 0.0f;
        if (c < cols)
#pragma unroll 8
            for (int k = wave; k < chunks; k += waves) v += sums[(size_t)k * cols + c];
        held[wave][threadIdx.x & 63] = v;
        __syncthreads();
        if (wave != 0 || c >= cols) return;
        for (int w = 1; w < waves; ++w) v += held[w][c & 63];
        if (n_active < n) {
            const int s = n_active ? place_of(active, n_active, c) : 0;
            if (!(s < n_active && active[s] == c)) v *= act_slope(bias ? bias[c] : 0.0f, act);
        }
        float* const to = c < n ? first : second;
        if (to) to[c < n ? c : c - n] = v;
    }
};
__global__ __launch_bounds__(256) void k_sum_chunks(SumChunks s) {
    __shared__ unsigned char held[4 * 64 * sizeof(float)];
    int group = blockIdx.x;
    if (blockIdx.y) group += (int)(blockIdx.y * gridDim.x);
    s(held, group);
}

template <typename T>
struct PlainOut {
    static constexpr bool kListed = false;
    T* y;
    int N;
    template <int V> __device__ void start(int, int) {}
    template <int V> __device__ void row(int m, int c, int valid, float (&v)[V]) { store_values<T, V, true>(y + (size_t)m * N + c, v, valid); }
};
// Rows [0, n) to one matrix, [padded, padded + n) to a second; nullptr: not wanted
template <typename T>
struct TwoOut {
    static constexpr bool kListed = false;
    T *first, *second;
    int N, n, padded;
    template <int V> __device__ void start(int, int) {}
    template <int V> __device__ void row(int m, int c, int valid, float (&v)[V]) {
        const bool behind = m >= padded;
        const int r = behind ? m - padded : m;
        T* const to = behind ? second : first;
        if (r < n && to) store_values<T, V, true>(to + (size_t)r * N + c, v, valid);
    }
};

// What a backward pass takes of the workspace
struct BwdPlan {
    int chunk_rows, chunks;
    DensePlans products;
    size_t dz_bytes, sum_bytes, dx_part_bytes, bytes;   // in this order, the parts of dW's product last
};
static size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }
enum class DzPass { kPlain, kListed, kPair };
// cols: columns of dz in a row, padding included (kPair: of dg and du, a thread takes the same ones of both); K: what dx's product sums over; dW_rows: rows of the weight gradients' product; sum_cols: columns of
// the sums
static BwdPlan plan_bwd(DzPass pass, int B, int d_in, long long cols, long long K, long long dW_rows, long long sum_cols, size_t elem) {
    BwdPlan p{};
    const bool f32 = elem == 4, direct = d_in % (16 / (int)elem) == 0;

    // About 4096 workgroups of k_dz_linear, whatever the width (gradients of a layer 256 -> 4096, fp32 at 2048 rows, 81.8 us against 87.3 with 2048, bf16 at 8192 rows 90.8 and 91.8, 256 -> 16384 at 2048 rows 87.7 and
    // 86.8, 256 -> 3001 at 4096 45.3 and 44.4), 2048 of the others (a fifth of 16384 neurons ablated, 4096 -> 16384 at 2048 rows, 476 us against 495 with 4096); two to eight rows to a thread and more only where the
    // grid would be too large
    const long long per_group = kDzCols * 16 / (long long)elem, groups = std::max(1ll, (cols / (pass == DzPass::kPair ? 2 : 1) + per_group - 1) / per_group);
    long long rows = std::min<long long>(8, std::max<long long>(2, B * groups / ((pass == DzPass::kPlain ? 4096 : 2048) * kDzRows))) * kDzRows;
    rows = std::max<long long>(rows, ((long long)B + 65534) / 65535);
    p.chunk_rows = (int)std::min<long long>(rows, kMaxSide);
    p.chunks = (int)((B + (long long)p.chunk_rows - 1) / p.chunk_rows);
    p.dz_bytes = whole((size_t)B * cols * elem);
    p.sum_bytes = whole((size_t)p.chunks * sum_cols * sizeof(float));
    const auto stages = [&](long long K) { return f32 ? stages_of<float>(K) : stages_of<uint16_t>(K); };
    p.products = plan_gradients(B, d_in, stages(K), (int)dW_rows, stages(B), f32, direct);
    p.dx_part_bytes = whole(part_bytes(p.products.dx, B, d_in, false));
    p.bytes = p.dz_bytes + p.sum_bytes + p.dx_part_bytes + whole(part_bytes(p.products.dW, (int)dW_rows, d_in, false));
    return p;
}

template <typename T, class P, class Q>
static srigl_status launch_gradients(const DensePlans& plans, const P& of_x, bool want_x, const Q& of_W, bool want_W, const SumChunks& sums, hipStream_t st) {
    if (want_x && want_W && plans.together && of_x.M > 0 && of_W.M > 0) return launch_dense_two<T>(of_x, of_W, sums, plans.dx.tile, st);
    if (sums.groups() > 0) {
        const GridLayers grid = grid_layers(sums.groups(), 256);
        hipLaunchKernelGGL(k_sum_chunks, dim3(grid.x, grid.times), dim3(256), 0, st, sums);
    }
    if (hip_ok(hipGetLastError()) != SRIGL_OK) return SRIGL_ERR_HIP;
    const srigl_status rc = want_x ? launch_dense<T, false>(of_x, plans.dx.tile, st) : SRIGL_OK;
    return rc == SRIGL_OK && want_W ? launch_dense<T, false>(of_W, plans.dW.tile, st) : rc;
}

template <typename T, typename TY>
static srigl_status linear_bwd(const BwdPlan& p, const void* dy, const void* x, int B, int d_in, const void* Wd, const int32_t* active, int n, const float* bias,
                               const void* z, int d_out, int act, void* dx, void* dWd, float* dbias, unsigned char* ws, hipStream_t st) {
    const int pitch = (int)padded(n);
    T* const dz = reinterpret_cast<T*>(ws);
    float *const sums = reinterpret_cast<float*>(ws + p.dz_bytes), *const dx_part = reinterpret_cast<float*>(ws + p.dz_bytes + p.sum_bytes), *const dW_part = reinterpret_cast<float*>(ws + p.dz_bytes + p.sum_bytes + p.dx_part_bytes);
    // without an activation or ablated neurons dz is dy: only its column sums are left to do
    const bool as_it_is = std::is_same<T, TY>::value && act == SRIGL_ACT_NONE && n == d_out && n % kPiece<T> == 0 && !astray(16, {dy});
    const bool listed = n < d_out;
    if (p.chunks > 0 && d_out > 0 && (n > 0 || dbias) && (!as_it_is || dbias)) {
        constexpr int COLS = kDzCols * kPiece<T>;
        T* const to = as_it_is || n == 0 ? nullptr : dz;
        float* const sum_to = dbias ? sums : nullptr;
        if (listed)
            hipLaunchKernelGGL((k_dz_listed<T, TY>), dim3((unsigned)std::max(1, (pitch + COLS - 1) / COLS), (unsigned)p.chunks), dim3(256), 0, st, (const TY*)dy, (const T*)z, active, n, B, d_out, act, to, pitch,
                               sum_to, p.chunk_rows);
        else
            hipLaunchKernelGGL((k_dz_linear<T, TY>), dim3((unsigned)((pitch + COLS - 1) / COLS), (unsigned)p.chunks), dim3(256), 0, st, (const TY*)dy, (const T*)z, n, B, act, to, pitch, sum_to,
                               p.chunk_rows);
    }
    const T* const d = as_it_is ? (const T*)dy : dz;
    const int d_pitch = as_it_is ? n : pitch;
    if (hip_ok(hipGetLastError()) != SRIGL_OK) return SRIGL_ERR_HIP;
    const DenseProduct<RowsOf<T>, ColsOf<T>, PlainOut<T>> of_x{{d, d_pitch, B - 1, d_pitch}, {(const T*)Wd, d_in, d_in, n}, {(T*)dx, d_in}, B, d_in, stages_of<T>(n), p.products.dx.parts, dx_part};
    const DenseProduct<ColsOf<T>, ColsOf<T>, PlainOut<T>> of_W{{d, d_pitch, d_pitch, B}, {(const T*)x, d_in, d_in, B}, {(T*)dWd, d_in}, n, d_in, stages_of<T>(B), p.products.dW.parts, dW_part};
    return launch_gradients<T>(p.products, of_x, dx != nullptr, of_W, dWd != nullptr, SumChunks{sums, p.chunks, d_out, d_out, active, n, bias, act, dbias, nullptr}, st);
}

template <typename T>
static srigl_status gated_bwd(const BwdPlan& p, const void* dh, const void* x, int B, int d_in, const void* Wg, const void* Wu, int n, const void* g, const void* u,
                              int act, void* dx, void* dWg, void* dWu, float* dbias_g, float* dbias_u, unsigned char* ws, hipStream_t st) {
    const int pitch = (int)padded(n);
    T* const dz = reinterpret_cast<T*>(ws);
    float *const sums = reinterpret_cast<float*>(ws + p.dz_bytes), *const dx_part = reinterpret_cast<float*>(ws + p.dz_bytes + p.sum_bytes), *const dW_part = reinterpret_cast<float*>(ws + p.dz_bytes + p.sum_bytes + p.dx_part_bytes);
    const bool want_sums = dbias_g || dbias_u;
    if (p.chunks > 0 && n > 0)
        hipLaunchKernelGGL(k_dz_gated<T>, dim3((unsigned)((pitch + kDzCols * kPiece<T> - 1) / (kDzCols * kPiece<T>)), (unsigned)p.chunks), dim3(256), 0, st, (const T*)dh, (const T*)g, (const T*)u, n, B, act, dz,
                           pitch, want_sums ? sums : nullptr, p.chunk_rows);
    if (hip_ok(hipGetLastError()) != SRIGL_OK) return SRIGL_ERR_HIP;
    const DenseProduct<RowsOf<T>, PairedCols<T>, PlainOut<T>> of_x{{dz, 2ll * pitch, B - 1, 2 * pitch}, {(const T*)Wg, bytes_between(Wg, Wu), d_in, d_in, n, pitch}, {(T*)dx, d_in}, B, d_in,
                                                                  stages_of<T>(2ll * pitch), p.products.dx.parts, dx_part};
    const DenseProduct<ColsOf<T>, ColsOf<T>, TwoOut<T>> of_W{{dz, 2ll * pitch, 2 * pitch, B}, {(const T*)x, d_in, d_in, B}, {(T*)dWg, (T*)dWu, d_in, n, pitch}, 2 * pitch, d_in, stages_of<T>(B),
                                                            p.products.dW.parts, dW_part};
    return launch_gradients<T>(p.products, of_x, dx != nullptr, of_W, dWg || dWu, SumChunks{sums, p.chunks, 2 * n, n, nullptr, n, nullptr, act, dbias_g, dbias_u}, st);
}

static bool bwd_sizes_fit(int B, int d_in, int d_out) { return B <= kMaxSide && d_in <= kMaxSide && d_out <= kMaxSide / 2; }

}  // namespace srigl

using namespace srigl;

extern "C" {

size_t srigl_structured_bwd_workspace_bytes(int32_t B, int32_t d_in, int32_t n_active, int32_t d_out, srigl_dtype dtype) {
    if (B < 0 || d_in < 0 || n_active < 0 || d_out < n_active || !known_dtype(dtype) || !bwd_sizes_fit(B, d_in, d_out)) return 0;
    return plan_bwd(n_active < d_out ? DzPass::kListed : DzPass::kPlain, B, d_in, padded(n_active), n_active, n_active, d_out, dtype_bytes(dtype)).bytes;
}

srigl_status srigl_structured_linear_bwd(const void* dy, srigl_dtype dy_dtype, const void* x, srigl_dtype x_dtype, int32_t B, int32_t d_in, const void* Wd,
                                         srigl_dtype w_dtype, const int32_t* active, int32_t n_active, const float* bias, const void* z, int32_t d_out,
                                         srigl_activation act, void* dx, void* dWd, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || d_in < 0 || n_active < 0 || d_out < 0 || n_active > d_out) return SRIGL_ERR_INVALID_ARG;
    if (!known_dtype(dy_dtype) || !known_dtype(x_dtype) || !known_dtype(w_dtype) || !known_act(act)) return SRIGL_ERR_INVALID_ARG;
    if (x_dtype != w_dtype || (dy_dtype != x_dtype && dy_dtype != SRIGL_F32) || !bwd_sizes_fit(B, d_in, d_out)) return SRIGL_ERR_UNSUPPORTED;
    if (active == nullptr && n_active != d_out && n_active != 0) return SRIGL_ERR_INVALID_ARG;
    const bool rows = B > 0 && n_active > 0;   // there is a product
    if (B > 0 && d_out > 0 && dy == nullptr && (dx || dWd || dbias)) return SRIGL_ERR_INVALID_ARG;
    if (rows && d_in > 0 && ((dx && Wd == nullptr) || (dWd && x == nullptr))) return SRIGL_ERR_INVALID_ARG;
    if (rows && act != SRIGL_ACT_NONE && z == nullptr && (dx || dWd || dbias)) return SRIGL_ERR_INVALID_ARG;
    if (astray(dtype_bytes(x_dtype), {x, Wd, z, dx, dWd}) || astray(dtype_bytes(dy_dtype), {dy}) || astray(4, {bias, active, dbias})) return SRIGL_ERR_INVALID_ARG;
    if (!dx && !dWd && !dbias) return SRIGL_OK;
    const BwdPlan p = plan_bwd(n_active < d_out ? DzPass::kListed : DzPass::kPlain, B, d_in, padded(n_active), n_active, n_active, d_out, dtype_bytes(x_dtype));
    if (p.bytes > 0 && workspace == nullptr) return SRIGL_ERR_CAPACITY;
    if (workspace_bytes < p.bytes) return SRIGL_ERR_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return SRIGL_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    if (d_in == 0) dx = dWd = nullptr;
    if (x_dtype == SRIGL_F32) return linear_bwd<float, float>(p, dy, x, B, d_in, Wd, active, n_active, bias, z, d_out, act, dx, dWd, dbias, ws, st);
    if (dy_dtype == SRIGL_F32) return linear_bwd<uint16_t, float>(p, dy, x, B, d_in, Wd, active, n_active, bias, z, d_out, act, dx, dWd, dbias, ws, st);
    return linear_bwd<uint16_t, uint16_t>(p, dy, x, B, d_in, Wd, active, n_active, bias, z, d_out, act, dx, dWd, dbias, ws, st);
}

size_t srigl_gated_bwd_workspace_bytes(int32_t B, int32_t d_in, int32_t n, srigl_dtype dtype) {
    if (B < 0 || d_in < 0 || n < 0 || !known_dtype(dtype) || !bwd_sizes_fit(B, d_in, n)) return 0;
    return plan_bwd(DzPass::kPair, B, d_in, 2 * padded(n), 2 * padded(n), 2 * padded(n), 2ll * n, dtype_bytes(dtype)).bytes;
}

srigl_status srigl_gated_linear_bwd(const void* dh, const void* x, srigl_dtype x_dtype, int32_t B, int32_t d_in, const void* Wg, const void* Wu, srigl_dtype w_dtype,
                                    int32_t n, const void* g, const void* u, srigl_activation act, void* dx, void* dWg, void* dWu, float* dbias_g, float* dbias_u,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || d_in < 0 || n < 0 || !known_dtype(x_dtype) || !known_dtype(w_dtype) || !known_act(act)) return SRIGL_ERR_INVALID_ARG;
    if (x_dtype != w_dtype || !bwd_sizes_fit(B, d_in, n)) return SRIGL_ERR_UNSUPPORTED;
    const bool any = dx || dWg || dWu || dbias_g || dbias_u, rows = B > 0 && n > 0;
    if (any && rows && (dh == nullptr || g == nullptr || u == nullptr)) return SRIGL_ERR_INVALID_ARG;
    if (rows && d_in > 0 && ((dx && (Wg == nullptr || Wu == nullptr)) || ((dWg || dWu) && x == nullptr))) return SRIGL_ERR_INVALID_ARG;
    if (astray(dtype_bytes(x_dtype), {dh, x, Wg, Wu, g, u, dx, dWg, dWu}) || astray(4, {dbias_g, dbias_u})) return SRIGL_ERR_INVALID_ARG;
    if (!any) return SRIGL_OK;
    const BwdPlan p = plan_bwd(DzPass::kPair, B, d_in, 2 * padded(n), 2 * padded(n), 2 * padded(n), 2ll * n, dtype_bytes(x_dtype));
    if (workspace_bytes < p.bytes || (p.bytes > 0 && workspace == nullptr)) return SRIGL_ERR_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return SRIGL_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    if (d_in == 0) dx = dWg = dWu = nullptr;
    if (x_dtype == SRIGL_F32) return gated_bwd<float>(p, dh, x, B, d_in, Wg, Wu, n, g, u, act, dx, dWg, dWu, dbias_g, dbias_u, ws, st);
    return gated_bwd<uint16_t>(p, dh, x, B, d_in, Wg, Wu, n, g, u, act, dx, dWg, dWu, dbias_g, dbias_u, ws, st);
}

}  // extern "C"
