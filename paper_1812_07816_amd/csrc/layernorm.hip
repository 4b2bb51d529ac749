// Layer normalisation over the C channels of each row (voxel or token), with a scale and a shift:
//   xhat = (x - mean) * rstd,  rstd = 1 / sqrt(var + eps) (biased variance),  y = gamma * xhat + beta.
// Backward, from x and the row's (mean, rstd), with g = dy * gamma:
//   dx = rstd * (g - mean_c(g) - xhat * mean_c(g * xhat)) (+ add),  dgamma = sum_rows dy * xhat,  dbeta = sum_rows dy.
//
// Bound: HBM.  A row stays in the registers of L lanes, K pieces of V values each, so that it is read once and the
// variance is a sum of squared differences from the mean (no cancellation where the mean is large); sums in fp32.  The
// sums over rows are kept per lane (a lane always has the same channels), added over the lanes of a workgroup in lane
// order, and over the workgroups in double in index order by a second launch (bit-reproducible).
#include "mi3d_internal.h"
#include "rows_common.h"

namespace mi3d {
namespace {

// Sum over the L lanes of a row; every lane gets it, with the same bits.  L > 64: the rows of a workgroup's only row, over
// `red` (16 floats a call, two calls alternate).
__device__ __forceinline__ float row_sum(float v, int L, float* red) {
    for (int o = 1; o < L && o < 64; o <<= 1) v += __shfl_xor(v, o);
    if (L > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        const int first = wave & ~(L / 64 - 1);
        v = 0.f;
        for (int w = 0; w < L / 64; ++w) v += red[first + w];
    }
    return v;
}

template <typename T, int V, int K>
__global__ void __launch_bounds__(512) ln_fwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                     T* y, float2* __restrict__ stats, long long rows, int C, int L, float eps) {
    __shared__ float red[16];
    const int l = threadIdx.x & (L - 1), mine = threadIdx.x / L, per = blockDim.x / L, P = C / V;
    const float inv = 1.f / (float)C;
    float ga[K][V], be[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (l + k * L < P) {
            load_values<float, V>(gamma + (l + k * L) * V, ga[k]);
            load_values<float, V>(beta + (l + k * L) * V, be[k]);
        }
    const long long step = (long long)gridDim.x * per;
    // (the lanes of a workgroup take the same number of turns: row_sum may wait for all of them)
    for (long long r0 = (long long)blockIdx.x * per; r0 < rows; r0 += step) {
        const long long r = r0 + mine;
        float v[K][V] = {}, s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r < rows && l + k * L < P) {
                load_values<T, V>(x + r * C + (l + k * L) * V, v[k]);
#pragma unroll
                for (int j = 0; j < V; ++j) s += v[k][j];
            }
        const float mean = row_sum(s, L, red) * inv;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v[k][j] -= mean;
                    s = fmaf(v[k][j], v[k][j], s);
                }
        const float rstd = 1.f / sqrtf(row_sum(s, L, red + 8) * inv + eps);
        if (r >= rows) continue;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = fmaf(v[k][j] * rstd, ga[k][j], be[k][j]);
                store_values<T, V>(y + r * C + (l + k * L) * V, o);
            }
        if (l == 0 && stats) stats[r] = float2{mean, rstd};
    }
}

// part: [workgroup][2][C], the workgroup's sums of dy * xhat and of dy
template <typename T, int V, int K>
__global__ void __launch_bounds__(512) ln_bwd_kernel(const T* dy, const T* x, const float2* __restrict__ stats, const float* __restrict__ gamma,
                                                     const T* add, T* dx, float* __restrict__ part, long long rows, int C, int L) {
    extern __shared__ float sums[];      // [rows of a turn][C]
    __shared__ float red[16];
    const int l = threadIdx.x & (L - 1), mine = threadIdx.x / L, per = blockDim.x / L, P = C / V;
    const float inv = 1.f / (float)C;
    float ga[K][V], dg[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (l + k * L < P) load_values<float, V>(gamma + (l + k * L) * V, ga[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[k][j] = db[k][j] = 0.f;
    }
    const long long step = (long long)gridDim.x * per;
    for (long long r0 = (long long)blockIdx.x * per; r0 < rows; r0 += step) {
        const long long r = r0 + mine;
        float xh[K][V] = {}, g[K][V] = {}, s1 = 0.f, s2 = 0.f;
        float2 st = {0.f, 0.f};
        if (r < rows) st = stats[r];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r < rows && l + k * L < P) {
                load_values<T, V>(x + r * C + (l + k * L) * V, xh[k]);
                load_values<T, V>(dy + r * C + (l + k * L) * V, g[k]);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    xh[k][j] = (xh[k][j] - st.x) * st.y;
                    dg[k][j] = fmaf(g[k][j], xh[k][j], dg[k][j]);
                    db[k][j] += g[k][j];
                    g[k][j] *= ga[k][j];
                    s1 += g[k][j];
                    s2 = fmaf(g[k][j], xh[k][j], s2);
                }
            }
        const float m1 = row_sum(s1, L, red) * inv, m2 = row_sum(s2, L, red + 8) * inv;
        if (r >= rows) continue;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P) {
                const long long at = r * C + (l + k * L) * V;
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = st.y * (g[k][j] - m1 - xh[k][j] * m2);
                if (add) {
                    float a[V];
                    load_values<T, V>(add + at, a);
#pragma unroll
                    for (int j = 0; j < V; ++j) o[j] += a[j];
                }
                store_values<T, V>(dx + at, o);
            }
    }
    float* out = part + (long long)blockIdx.x * 2 * C;
    for (int q = 0; q < 2; ++q) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P)
#pragma unroll
                for (int j = 0; j < V; ++j) (per > 1 ? sums + mine * C : out + q * C)[(l + k * L) * V + j] = q ? db[k][j] : dg[k][j];
        __syncthreads();
        if (per > 1)
            for (int c = threadIdx.x; c < C; c += blockDim.x) {
                float s = 0.f;
                for (int i = 0; i < per; ++i) s += sums[i * C + c];
                out[q * C + c] = s;
            }
    }
}

// dgamma, dbeta from the workgroups' sums: 16 columns a workgroup, thread (slice, column) adds parts slice, slice + 16, ...
__global__ void __launch_bounds__(256) ln_finish_kernel(const float* __restrict__ part, int parts, int C, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double red[16][17];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    double s = 0.0;
    if (c < 2 * C)
        for (int p = slice; p < parts; p += 16) s += (double)part[(long long)p * 2 * C + c];
    red[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * C) {
        for (int i = 1; i < 16; ++i) s += red[i][col];
        (c < C ? dgamma[c] : dbeta[c - C]) = (float)s;
    }
}

// Lanes of a row (a power of two) and pieces of a lane, at most 4: of the ways that fit, the one with the fewest idle lanes, and of
// those the one with the most lanes.
struct Rows {
    int V, L, K;
};
bool rows_plan(int C, Rows* p) {
    if (C <= 0) return false;
    p->V = C % 8 ? 1 : 8;
    const int P = C / p->V;
    p->L = 0;
    for (int L = 1; L <= 512; L <<= 1) {
        const int K = (P + L - 1) / L;
        if (K <= 4 && (!p->L || L * K <= p->L * p->K)) { p->L = L; p->K = K; }
    }
    return p->L != 0;      // up to 2048 pieces
}
int threads_of(const Rows& p) { return p.L > 256 ? p.L : 256; }
constexpr int MOST_PARTS = 1024;
int parts_of(const Rows& p, size_t rows) {
    const long long turns = ((long long)rows + threads_of(p) / p.L - 1) / (threads_of(p) / p.L);
    return (int)(turns < MOST_PARTS ? turns : MOST_PARTS);
}

template <typename T>
int ln_fwd(const void* x, const float* gamma, const float* beta, size_t rows, int C, float eps, void* y, float* stats, void* stream) {
    Rows p;
    if (rows == 0 && C > 0) return rows_plan(C, &p) ? MI3D_OK : MI3D_ERR_UNSUPPORTED;
    if (C <= 0 || !x || !gamma || !beta || !y || !(eps >= 0.f)) return MI3D_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(gamma) || !aligned16(beta) || !aligned16(y) || ((uintptr_t)stats & 7)) return MI3D_ERR_INVALID_ARG;
    if (!rows_plan(C, &p) || rows >= (1ull << 40)) return MI3D_ERR_UNSUPPORTED;
    const int threads = threads_of(p);
    const long long turns = ((long long)rows + threads / p.L - 1) / (threads / p.L);
    const unsigned grid = (unsigned)(turns < 4096 ? turns : 4096);
    auto go = [&](auto kernel) { kernel<<<grid, threads, 0, (hipStream_t)stream>>>((const T*)x, gamma, beta, (T*)y, (float2*)stats, (long long)rows, C, p.L, eps); };
    switch (p.V + p.K) {
        case 2: go(ln_fwd_kernel<T, 1, 1>); break;
        case 3: go(ln_fwd_kernel<T, 1, 2>); break;
        case 4: go(ln_fwd_kernel<T, 1, 3>); break;
        case 5: go(ln_fwd_kernel<T, 1, 4>); break;
        case 9: go(ln_fwd_kernel<T, 8, 1>); break;
        case 10: go(ln_fwd_kernel<T, 8, 2>); break;
        case 11: go(ln_fwd_kernel<T, 8, 3>); break;
        default: go(ln_fwd_kernel<T, 8, 4>); break;
    }
    return check_launch();
}

template <typename T>
int ln_bwd(const void* dy, const void* x, const float* stats, const float* gamma, const void* add, size_t rows, int C, void* dx, float* dgamma,
           float* dbeta, void* ws, size_t ws_bytes, void* stream) {
    Rows p;
    if (C <= 0 || !gamma || !dgamma || !dbeta || !aligned16(gamma)) return MI3D_ERR_INVALID_ARG;
    if (rows && (!dy || !x || !stats || !dx || !ws)) return MI3D_ERR_INVALID_ARG;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(add) || !aligned16(dx) || !aligned16(ws) || ((uintptr_t)stats & 7)) return MI3D_ERR_INVALID_ARG;
    if (!rows_plan(C, &p) || rows >= (1ull << 40)) return MI3D_ERR_UNSUPPORTED;
    if (ws_bytes < mi3d_layernorm_workspace_bytes(rows, C)) return MI3D_ERR_WORKSPACE;
    const int threads = threads_of(p), parts = parts_of(p, rows);
    if (parts) {
        auto go = [&](auto kernel) {
            const int per = threads / p.L;
            kernel<<<parts, threads, per > 1 ? (size_t)per * C * sizeof(float) : 0, (hipStream_t)stream>>>(      // (at most 32 KB)
                (const T*)dy, (const T*)x, (const float2*)stats, gamma, (const T*)add, (T*)dx, (float*)ws, (long long)rows, C, p.L);
        };
        switch (p.V + p.K) {
            case 2: go(ln_bwd_kernel<T, 1, 1>); break;
            case 3: go(ln_bwd_kernel<T, 1, 2>); break;
            case 4: go(ln_bwd_kernel<T, 1, 3>); break;
            case 5: go(ln_bwd_kernel<T, 1, 4>); break;
            case 9: go(ln_bwd_kernel<T, 8, 1>); break;
            case 10: go(ln_bwd_kernel<T, 8, 2>); break;
            case 11: go(ln_bwd_kernel<T, 8, 3>); break;
            default: go(ln_bwd_kernel<T, 8, 4>); break;
        }
        const int st = check_launch();
        if (st) return st;
    }
    ln_finish_kernel<<<(2 * C + 15) / 16, 256, 0, (hipStream_t)stream>>>((const float*)ws, parts, C, dgamma, dbeta);
    return check_launch();
}

}  // namespace
}  // namespace mi3d

using namespace mi3d;

extern "C" {

size_t mi3d_layernorm_workspace_bytes(size_t rows, int C) {
    Rows p;
    return rows_plan(C, &p) ? (size_t)parts_of(p, rows) * 2 * C * sizeof(float) : 0;
}

int mi3d_layernorm_fwd(const void* x, const float* gamma, const float* beta, size_t rows, int C, float eps, void* y, float* stats, void* stream) {
    return ln_fwd<uint16_t>(x, gamma, beta, rows, C, eps, y, stats, stream);
}
int mi3d_layernorm_fwd_f32(const void* x, const float* gamma, const float* beta, size_t rows, int C, float eps, void* y, float* stats, void* stream) {
    return ln_fwd<float>(x, gamma, beta, rows, C, eps, y, stats, stream);
}
int mi3d_layernorm_bwd(const void* dy, const void* x, const float* stats, const float* gamma, const void* add, size_t rows, int C, void* dx,
                       float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
    return ln_bwd<uint16_t>(dy, x, stats, gamma, add, rows, C, dx, dgamma, dbeta, ws, ws_bytes, stream);
}
int mi3d_layernorm_bwd_f32(const void* dy, const void* x, const float* stats, const float* gamma, const void* add, size_t rows, int C, void* dx,
                           float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
    return ln_bwd<float>(dy, x, stats, gamma, add, rows, C, dx, dgamma, dbeta, ws, ws_bytes, stream);
}

}  // extern "C"
