// The gated feed-forward block's forward products for few rows (single tokens and small batches of them):
//   out[m][n] = sum_k x[m][k] w[n][k],  or  act(g) * u of two such sums.
//
// Bound: the bytes of the weights, of which every one is used for at most 64 rows (small matrices of more rows: the latency of
// one pass over k, which the waves of a workgroup share); so they go from memory to registers, in the
// layout of the matrix instructions (16 rows of w by 16 rows of x), without LDS: a lane takes 32 of the 128 bytes of k that
// four lanes read of a row of w, and the same k of x, whose order inside a sum does not matter as long as both have the same.  A
// workgroup serves 16 columns n and up to 64 rows m; its waves take every W-th 128 bytes of k each and their sums are added in wave order.
// bf16: v_mfma_f32_16x16x32_bf16, fp32: v_mfma_f32_16x16x4_f32.
#include "ffn.h"

namespace mi3d {
namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

template <typename T>
__device__ __forceinline__ f32x4 product(const uint4& w, const uint4& x, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
    } else {
        const uint32_t a[4] = {w.x, w.y, w.z, w.w}, b[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, a[j]), __builtin_bit_cast(float, b[j]), c, 0, 0, 0);
        return c;
    }
}

// NB blocks of 16 rows of x; U pieces of 128 bytes of k requested ahead of their products
template <typename T, int NB, bool GATED, int ACT, int U>
__global__ void __launch_bounds__(512) few_rows_kernel(const T* __restrict__ x, const T* __restrict__ w, long long rows, int K, int N,
                                                        T* __restrict__ out, T* __restrict__ gu) {
    constexpr int G = GATED ? 2 : 1, E = sizeof(T), PIECE = 128 / E;
    extern __shared__ f32x4 sums[];      // [wave][G * NB][lane]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6;
    const int r = lane & 15, part = lane >> 4, n0 = blockIdx.x * 16;
    const long long m0 = (long long)blockIdx.y * 16 * NB;
    x += m0 * K;
    rows = rows - m0 < 16 * NB ? (int)(rows - m0) : 16 * NB;
    out += m0 * N;
    if (GATED && gu) gu += m0 * 2 * N;
    const bool has_w = n0 + r < N;
    const T* wp = w + (long long)(has_w ? n0 + r : 0) * K + part * (PIECE / 4);
    const T* xp = x + part * (PIECE / 4);
    const long long up = (long long)N * K;
    f32x4 acc[G][NB];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[g][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint4 zero = {0, 0, 0, 0};
    for (int k0 = wave * PIECE; k0 < K; k0 += W * PIECE * U) {
        uint4 vw[U][G][2], vx[U][NB][2];
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int k = k0 + i * W * PIECE, at = k + q * (16 / E);
                const bool in = at + part * (PIECE / 4) < K;      // (a piece of 16 bytes lies inside a row or outside)
#pragma unroll
                for (int g = 0; g < G; ++g) vw[i][g][q] = in && has_w ? *(const uint4*)(wp + g * up + at) : zero;
#pragma unroll
                for (int b = 0; b < NB; ++b) vx[i][b][q] = in && 16 * b + r < rows ? *(const uint4*)(xp + (long long)(16 * b + r) * K + at) : zero;
            }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int b = 0; b < NB; ++b) acc[g][b] = product<T>(vw[i][g][q], vx[i][b][q], acc[g][b]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int b = 0; b < NB; ++b) sums[(wave * G * NB + g * NB + b) * 64 + lane] = acc[g][b];
    __syncthreads();
    // lane l of a block: row l % 16, columns 4 (l / 16) .. + 3
    for (int e = threadIdx.x; e < NB * 64; e += blockDim.x) {
        const int b = e >> 6, m = 16 * b + (e & 15), n = n0 + 4 * (e >> 4 & 3);
        if (m >= rows || n >= N) continue;
        f32x4 v[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            v[g] = sums[(g * NB + b) * 64 + (e & 63)];
            for (int i = 1; i < W; ++i) {
                const f32x4 o = sums[(i * G * NB + g * NB + b) * 64 + (e & 63)];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[g][j] += o[j];
            }
        }
        auto put = [&](T* p, const f32x4& f) {
            if constexpr (E == 2) *(uint2*)p = uint2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
            else *(f32x4*)p = f;
        };
        if constexpr (GATED) {
            if (gu) {
                put(gu + (long long)m * 2 * N + n, v[0]);
                put(gu + (long long)m * 2 * N + N + n, v[1]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[0][j] = activation<T, ACT>(v[0][j]) * v[1][j];
        }
        put(out + (long long)m * N + n, v[0]);      // (GATED: h, rounded to its type for the second product, as on tiles)
    }
}

}  // namespace

// Blocks of 16 rows of a workgroup: as many (up to 4) as leave a workgroup for every compute unit
// (64 x 4096 -> 1024: 20.1 us with 4, 13.2 with 2, 9.4 with 1; fp32, 1331 x 200 -> 2 x 520: 17.0, 19.2 and 24.8).  Fewer than 16 x 256 columns
// of one block of rows leave units idle all the same, as no workgroup takes a part of k: one row of 4096 -> 1024, 64 workgroups, takes 7.1 us for
// 8.4 MB, 1024 -> 2 x 4096, 256 workgroups, 6.5 us for 16.8 MB.
static int blocks_of(long long rows, int N) {
    const long long cols = (N + 15) / 16;
    int nb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    while (nb > 1 && cols * ((rows + 16 * nb - 1) / (16 * nb)) < cu_count()) nb /= 2;
    return nb;
}

// What it is expected to take, in microseconds: for every workgroup of a compute unit (one where there are fewer workgroups than units) a
// fixed time and one for each 128 bytes of k, measured
// with 1, 2 and 4 blocks of rows on the sizes above and one row of 1024 and 4096
double few_rows_us(bool bf16, long long rows, long long K, long long N) {
    const int nb = blocks_of(rows, (int)N);
    const double groups = (double)((N + 15) / 16) * (double)((rows + 16 * nb - 1) / (16 * nb)) / cu_count(), pieces = (double)((K * (bf16 ? 2 : 4) + 127) / 128);
    const long long down = (rows + 16 * nb - 1) / (16 * nb), across = (N + 15) / 16;
    if (down > 65535 || down * across * 512 >= (1ll << 31)) return 1e30;      // (a launch's second dimension, and its threads of 8 waves each)
    static constexpr double each[2][3] = {{0.12, 0.30, 0.60}, {0.09, 0.22, 0.40}};
    return 3.5 + (groups < 1.0 ? 1.0 : groups) * ((bf16 ? 0.2 : 0.8) + pieces * each[bf16][nb / 2]);
}

int few_rows_product(bool bf16, bool gated, const void* x, const void* w, long long rows, int K, int N, int act, void* out, void* gu, hipStream_t s) {
    const int e = bf16 ? 2 : 4, pieces = (K * e + 127) / 128, nb = blocks_of(rows, N);
    // waves of a workgroup: two pieces each where that takes no more than 8 (16 are slower: 19.0 and 15.1 us for 1331 x 520 -> 200 in fp32)
    int W = 1;
    while (W < 8 && 2 * W < pieces) W *= 2;
    const dim3 grid((unsigned)((N + 15) / 16), (unsigned)((rows + 16 * nb - 1) / (16 * nb)));
    const size_t lds = (size_t)W * (gated ? 2 : 1) * nb * 1024;
    auto go = [&](auto type, auto kernel) {
        typedef decltype(type) T;
        kernel<<<grid, 64 * W, lds, s>>>((const T*)x, (const T*)w, rows, K, N, (T*)out, (T*)gu);
    };
    constexpr int SILU = MI3D_ACT_SILU, GELU = MI3D_ACT_GELU;
    auto pick = [&](auto type) {
        typedef decltype(type) T;
        if (!gated) {
            if (nb == 1) go(type, few_rows_kernel<T, 1, false, SILU, 4>);
            else if (nb == 2) go(type, few_rows_kernel<T, 2, false, SILU, 2>);
            else go(type, few_rows_kernel<T, 4, false, SILU, 2>);
        } else if (act == SILU) {
            if (nb == 1) go(type, few_rows_kernel<T, 1, true, SILU, 4>);
            else if (nb == 2) go(type, few_rows_kernel<T, 2, true, SILU, 2>);
            else go(type, few_rows_kernel<T, 4, true, SILU, 1>);
        } else {
            if (nb == 1) go(type, few_rows_kernel<T, 1, true, GELU, 4>);
            else if (nb == 2) go(type, few_rows_kernel<T, 2, true, GELU, 2>);
            else go(type, few_rows_kernel<T, 4, true, GELU, 1>);
        }
    };
    if (bf16) pick(uint16_t{});
    else pick(float{});
    return check_launch();
}

}  // namespace mi3d
