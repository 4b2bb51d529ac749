// Layer normalisation over the C channels of each row (voxel or token), with a scale and a shift:
//   xhat = (x - mean) * rstd,  rstd = 1 / sqrt(var + eps) (biased variance),  y = gamma * xhat + beta.
// Backward, from x and the row's (mean, rstd), with g = dy * gamma:
//   dx = rstd * (g - mean_c(g) - xhat * mean_c(g * xhat)) (+ add),  dgamma = sum_rows dy * xhat,  dbeta = sum_rows dy.
//
// Bound: HBM (bf16, 192^3 rows of 32: forward 189 us, backward with a second gradient 345 us = 5.25 TB/s of
// the tensors alone, 5.4 with the rows' statistics, where a copy reaches 5.1; 27648
// rows of 320: backward 20 us and 4 for the sums, fp32 31 and 5).  A row stays in the registers of L lanes, K pieces of eight values each, so that it is read once and the
// variance is a sum of squared differences from the mean (no cancellation where the mean is large); sums in fp32.  The
// sums over rows are kept per lane (a lane always has the same channels), added over the lanes of a workgroup in lane
// order, and over the workgroups in double in a fixed order by a second launch (bit-reproducible).  fp32 carries 108 rows of a lane and 64
// lanes at 192^3 rows of 32: 1e-5 of the sum of magnitudes at the very worst; sums in 64 bits
// would take twice the registers of a lane.
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

// How a row lies in pieces: EVEN: C in multiples of 8, aligned pieces of 8.  ODD: any other C from 8 on, pieces of 8 at any address, the
// last of them moved back to end with the row, so that its first `skip` values are the last ones of the piece before and count
// there (both lanes store the same).  TINY: C below 8, one value at a time.
enum Form { EVEN, ODD, TINY };
template <Form F> constexpr int V = F == TINY ? 1 : 8;
struct Place {
    int col, skip;
    __device__ __forceinline__ bool counts(int j) const { return j >= skip; }
};
template <Form F>
__device__ __forceinline__ Place place(int piece, int C) {
    const int at = piece * V<F>;
    if (F != ODD || at + 8 <= C) return Place{at, 0};
    return Place{C - 8, at + 8 - C};
}
template <Form F, typename T>
__device__ __forceinline__ void get(const T* p, float (&f)[V<F>]) {
    if constexpr (F == ODD) load8_anywhere(p, f);
    else load_values<T, V<F>>(p, f);
}
template <Form F, typename T>
__device__ __forceinline__ void put(T* p, const float (&f)[V<F>]) {
    if constexpr (F == ODD) store8_anywhere(p, f);
    else store_values<T, V<F>>(p, f);
}

template <typename T, Form F, int K>
__global__ void __launch_bounds__(512) ln_fwd_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                     T* y, float2* __restrict__ stats, long long rows, int C, int L, float eps) {
    __shared__ float red[16];
    const int l = threadIdx.x & (L - 1), mine = threadIdx.x / L, per = blockDim.x / L, P = (C + V<F> - 1) / V<F>;
    const float inv = 1.f / (float)C;
    float ga[K][V<F>], be[K][V<F>];
    Place at[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (l + k * L < P) {
            at[k] = place<F>(l + k * L, C);
            get<F>(gamma + at[k].col, ga[k]);
            get<F>(beta + at[k].col, be[k]);
        }
    const long long step = (long long)gridDim.x * per;
    // (the lanes of a workgroup take the same number of turns: row_sum may wait for all of them)
    for (long long r0 = (long long)blockIdx.x * per; r0 < rows; r0 += step) {
        const long long r = r0 + mine;
        float v[K][V<F>] = {}, s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r < rows && l + k * L < P) {
                get<F>(x + r * C + at[k].col, v[k]);
#pragma unroll
                for (int j = 0; j < V<F>; ++j) s += F != ODD || at[k].counts(j) ? v[k][j] : 0.f;
            }
        const float mean = row_sum(s, L, red) * inv;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P)
#pragma unroll
                for (int j = 0; j < V<F>; ++j) {
                    v[k][j] -= mean;
                    const float d = F != ODD || at[k].counts(j) ? v[k][j] : 0.f;
                    s = fmaf(d, d, s);
                }
        const float rstd = 1.f / sqrtf(row_sum(s, L, red + 8) * inv + eps);
        if (r >= rows) continue;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P) {
                float o[V<F>];
#pragma unroll
                for (int j = 0; j < V<F>; ++j) o[j] = fmaf(v[k][j] * rstd, ga[k][j], be[k][j]);
                put<F>(y + r * C + at[k].col, o);
            }
        if (l == 0 && stats) stats[r] = float2{mean, rstd};
    }
}

// part: [workgroup][2][C], the workgroup's sums of dy * xhat and of dy
template <typename T, Form F, int K>
__global__ void __launch_bounds__(512) ln_bwd_kernel(const T* dy, const T* x, const float2* __restrict__ stats, const float* __restrict__ gamma,
                                                     const T* add, T* dx, float* __restrict__ part, long long rows, int C, int L) {
    extern __shared__ float sums[];      // [rows of a turn][C]
    __shared__ float red[16];
    const int l = threadIdx.x & (L - 1), mine = threadIdx.x / L, per = blockDim.x / L, P = (C + V<F> - 1) / V<F>;
    const float inv = 1.f / (float)C;
    float ga[K][V<F>], dg[K][V<F>] = {}, db[K][V<F>] = {};
    Place at[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (l + k * L < P) {
            at[k] = place<F>(l + k * L, C);
            get<F>(gamma + at[k].col, ga[k]);
        }
    const long long step = (long long)gridDim.x * per;
    for (long long r0 = (long long)blockIdx.x * per; r0 < rows; r0 += step) {
        const long long r = r0 + mine;
        float xh[K][V<F>] = {}, g[K][V<F>] = {}, s1 = 0.f, s2 = 0.f;
        float2 st = {0.f, 0.f};
        if (r < rows) st = stats[r];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r < rows && l + k * L < P) {
                get<F>(x + r * C + at[k].col, xh[k]);
                get<F>(dy + r * C + at[k].col, g[k]);
#pragma unroll
                for (int j = 0; j < V<F>; ++j) {
                    xh[k][j] = (xh[k][j] - st.x) * st.y;
                    dg[k][j] = fmaf(g[k][j], xh[k][j], dg[k][j]);
                    db[k][j] += g[k][j];
                    g[k][j] *= ga[k][j];
                    const float d = F != ODD || at[k].counts(j) ? g[k][j] : 0.f;
                    s1 += d;
                    s2 = F != ODD || at[k].counts(j) ? fmaf(d, xh[k][j], s2) : s2;
                }
            }
        const float m1 = row_sum(s1, L, red) * inv, m2 = row_sum(s2, L, red + 8) * inv;
        // (an ODD row's pieces overlap: none is stored before all are read, add's among them, which dx may be)
        float a[K][V<F>] = {};
        if (add && r < rows) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (l + k * L < P) get<F>(add + r * C + at[k].col, a[k]);
        }
        if (F == ODD && L > 64) __syncthreads();
        if (r >= rows) continue;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P) {
                float o[V<F>];
#pragma unroll
                for (int j = 0; j < V<F>; ++j) o[j] = st.y * (g[k][j] - m1 - xh[k][j] * m2) + a[k][j];
                put<F>(dx + r * C + at[k].col, o);
            }
    }
    float* out = part + (long long)blockIdx.x * 2 * C;
    for (int q = 0; q < 2; ++q) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (l + k * L < P)
#pragma unroll
                for (int j = 0; j < V<F>; ++j)
                    if (F != ODD || at[k].counts(j)) (per > 1 ? sums + mine * C : out + q * C)[at[k].col + j] = q ? db[k][j] : dg[k][j];
        __syncthreads();
        if (per > 1)
            for (int c = threadIdx.x; c < C; c += blockDim.x) {
                float s = 0.f;
                for (int i = 0; i < per; ++i) s += sums[i * C + c];
                out[q * C + c] = s;
            }
    }
}

// dgamma, dbeta from the workgroups' sums: 16 columns a workgroup, thread (slice, column) adds parts slice, slice + 64, ... in double, and the
// slices are added in order.  Bound: the latency of the loads, of which four are under way (27648 x 320, 864 parts: 4 us; 25 with 16
// slices and one load at a time).
__global__ void __launch_bounds__(1024) ln_finish_kernel(const float* __restrict__ part, int parts, int C, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double red[64][17];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    double s = 0.0;
    if (c < 2 * C) {
        int p = slice;
        for (; p + 192 < parts; p += 256) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = part[(long long)(p + 64 * i) * 2 * C + c];
            s += (double)v[0] + (double)v[1] + (double)v[2] + (double)v[3];
        }
        for (; p < parts; p += 64) s += (double)part[(long long)p * 2 * C + c];
    }
    red[slice][col] = s;
    __syncthreads();
    for (int half = 32; half; half >>= 1) {
        if (slice < half) red[slice][col] += red[slice + half][col];
        __syncthreads();
    }
    if (slice == 0 && c < 2 * C) (c < C ? dgamma[c] : dbeta[c - C]) = (float)red[0][col];
}

// Lanes of a row (a power of two) and pieces of a lane, at most 4: of the ways that fit, the one with the fewest idle lanes, and of
// those the one with the most lanes; more than a wavefront's only where its lanes cannot hold the row.  Measured on 2^27 values,
// forward / backward in us, where a copy's rate makes 104 / 156 in bf16 and 208 / 313 in fp32:
//   channels (pieces)   lanes x pieces of a lane: bf16, fp32
//     56 (7)     8 x 1: 106 / 153, 222 / 301     4 x 2: 123 / 171, 279 / 395     2 x 4: 144 / 204, 353 / 470
//    200 (25)   32 x 1: 106 / 164, 231 / 307    16 x 2: 112 / 162, 234 / 344     8 x 4: 136 / 204, 253 / 345
//    320 (40)   16 x 3: 129 / 201, 202 / 339    32 x 2: 129 / 169, 212 / 311    64 x 1: 126 / 204, 230 / 290
//     24 (3)     1 x 3: 134 / 193, 355 / 506     2 x 2: 126 / 178, 295 / 424     4 x 1: 109 / 158, 227 / 311
//     72 (9)     4 x 3: 123 / 184, 297 / 442     8 x 2: 125 / 178, 242 / 351    16 x 1: 123 / 195, 236 / 306
// The rule takes the first of each line.  It is right where a lane then has one piece; rows of 3, 5, 6, 9 or 10 pieces are read in
// pieces of 16 or 32 bytes out of every 48 to 96, which costs more than idle lanes, most of all in fp32.
struct Rows {
    Form form;
    int L, K;
};
bool rows_plan(int C, Rows* p) {
    if (C <= 0 || C > 16384) return false;
    p->form = C < 8 ? TINY : C % 8 ? ODD : EVEN;
    const int P = C < 8 ? C : (C + 7) / 8, most = C < 8 ? 1 : 4;
    p->L = 0;
    for (int L = 1; L <= 512; L <<= 1) {      // (512 lanes of 4 pieces: 16384 values)
        const int K = (P + L - 1) / L;
        if (K <= most && (!p->L || (L <= 64 && L * K <= p->L * p->K))) { p->L = L; p->K = K; }
    }
    return true;
}
int threads_of(const Rows& p) { return p.L > 256 ? p.L : 256; }
// Workgroups of the backward pass: four for a compute unit, fewer of wide rows, whose registers leave room for two or one and whose sums
// are a part of the traffic; all with as many turns, but for one.  us with four, two and one, the second launch included (bf16): 8192 x 4096
// 61, 50, 70; 4096 x 16384 161, 121, 109; 27648 x 320 24, 21, 26 (few turns each: two would do there)
int parts_of(const Rows& p, size_t rows, int C) {
    const long long most = C <= 1024 ? 1024 : C <= 8192 ? 512 : 256;
    const long long per = threads_of(p) / p.L, turns = ((long long)rows + per - 1) / per, each = (turns + most - 1) / most;
    return (int)(each ? (turns + each - 1) / each : 0);
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
    if (p.form == TINY) go(ln_fwd_kernel<T, TINY, 1>);
    else if (p.form == EVEN) go(p.K == 1 ? ln_fwd_kernel<T, EVEN, 1> : p.K == 2 ? ln_fwd_kernel<T, EVEN, 2> : p.K == 3 ? ln_fwd_kernel<T, EVEN, 3> : ln_fwd_kernel<T, EVEN, 4>);
    else go(p.K == 1 ? ln_fwd_kernel<T, ODD, 1> : p.K == 2 ? ln_fwd_kernel<T, ODD, 2> : p.K == 3 ? ln_fwd_kernel<T, ODD, 3> : ln_fwd_kernel<T, ODD, 4>);
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
    const int threads = threads_of(p), parts = parts_of(p, rows, C);
    if (parts) {
        auto go = [&](auto kernel) {
            const int per = threads / p.L;
            kernel<<<parts, threads, per > 1 ? (size_t)per * C * sizeof(float) : 0, (hipStream_t)stream>>>(      // (at most 32 KB)
                (const T*)dy, (const T*)x, (const float2*)stats, gamma, (const T*)add, (T*)dx, (float*)ws, (long long)rows, C, p.L);
        };
        if (p.form == TINY) go(ln_bwd_kernel<T, TINY, 1>);
        else if (p.form == EVEN) go(p.K == 1 ? ln_bwd_kernel<T, EVEN, 1> : p.K == 2 ? ln_bwd_kernel<T, EVEN, 2> : p.K == 3 ? ln_bwd_kernel<T, EVEN, 3> : ln_bwd_kernel<T, EVEN, 4>);
        else go(p.K == 1 ? ln_bwd_kernel<T, ODD, 1> : p.K == 2 ? ln_bwd_kernel<T, ODD, 2> : p.K == 3 ? ln_bwd_kernel<T, ODD, 3> : ln_bwd_kernel<T, ODD, 4>);
        const int st = check_launch();
        if (st) return st;
    }
    ln_finish_kernel<<<(2 * C + 15) / 16, 1024, 0, (hipStream_t)stream>>>((const float*)ws, parts, C, dgamma, dbeta);
    return check_launch();
}

}  // namespace
}  // namespace mi3d

using namespace mi3d;

extern "C" {

size_t mi3d_layernorm_workspace_bytes(size_t rows, int C) {
    Rows p;
    return rows_plan(C, &p) ? (size_t)parts_of(p, rows, C) * 2 * C * sizeof(float) : 0;
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
