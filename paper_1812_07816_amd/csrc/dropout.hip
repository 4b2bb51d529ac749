// Dropout whose mask is never stored: the backward pass draws the same numbers again.
//
// Number i of the stream (seed, offset) is a 16-bit half of the output of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011) for the key `seed` and the counter (i / 8, offset): word
// (i % 8) / 2, low half first.  A value is kept where its number is below T = 65536 (1 - p), rounded to a whole number, and
// multiplied by 65536 / T: the expected value is exact for the probability that the comparison has, which is within 2^-17 of 1 - p.
// One draw of the generator serves the eight values that a thread moves at a time.
//
// Bound: HBM for the values; the generator's ten rounds (20 products of 32 by 32 bits) run beside the loads.  bf16, 192^3 x 32 with a
// residual: 272 us = 5.0 TB/s (a copy reaches 5.1); whole channels, 2 x 96^3 x 64: 84 us = 5.4 TB/s, out of the last cache in part.
#include <cmath>

#include "mi3d_internal.h"
#include "rows_common.h"

namespace mi3d {
namespace {

struct Stream {
    uint32_t key0, key1;
    uint64_t offset;
    const uint64_t* more;      // device memory, added to the offset (or null): a captured graph's replays differ by it
};

__device__ __forceinline__ uint4 philox(uint64_t i, uint64_t offset, uint32_t k0, uint32_t k1) {
    uint4 c = {(uint32_t)i, (uint32_t)(i >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = uint4{(uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}
__device__ __forceinline__ uint32_t number(const uint4& w, int j) {
    const uint32_t v = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
    return j & 1 ? v >> 16 : v & 0xFFFFu;
}
// bit j: value j of eight is kept
__device__ __forceinline__ uint32_t kept8(const uint4& w, uint32_t T) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m |= number(w, j) < T ? 1u << j : 0u;
    return m;
}

// out[i] = (kept ? a[i] * scale : 0) (+ res[i]); a dropped value is 0 whatever it was
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const T* a, const T* res, T* out, long long n, Stream s, uint32_t limit, float scale) {
    const uint64_t offset = s.offset + (s.more ? *s.more : 0);
    const long long groups = (n + 7) / 8, step = (long long)gridDim.x * 256;
    for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; g < groups; g += step) {
        const uint32_t m = kept8(philox((uint64_t)g, offset, s.key0, s.key1), limit);
        if (8 * g + 8 <= n) {
            float v[8], r[8];
            load_values<T, 8>(a + 8 * g, v);
            if (RES) load_values<T, 8>(res + 8 * g, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = m >> j & 1 ? v[j] * scale : 0.f;
                if (RES) v[j] += r[j];
            }
            store_values<T, 8>(out + 8 * g, v);
        } else {
            for (long long i = 8 * g; i < n; ++i) {
                float v[1], r[1] = {0.f};
                load_values<T, 1>(a + i, v);
                if (RES) load_values<T, 1>(res + i, r);
                v[0] = (m >> (i & 7) & 1 ? v[0] * scale : 0.f) + r[0];
                store_values<T, 1>(out + i, v);
            }
        }
    }
}

// Whole channels: value (n, v, c) of [N][voxels][C] goes by number n C + c.  A workgroup serves one sample: its bits lie in LDS,
// those of the first channels once more behind the last, so that eight values in a row, from any channel on, find theirs in two bytes.
template <typename T>
__global__ void __launch_bounds__(256) dropout_channels_kernel(const T* a, T* out, long long voxels, int C, Stream s, uint32_t limit, float scale) {
    extern __shared__ uint64_t bits[];
    const uint64_t offset = s.offset + (s.more ? *s.more : 0);
    const long long n = blockIdx.y;
    for (int j = threadIdx.x; j < (C + 16 + 255) / 256 * 256; j += 256) {
        const uint64_t i = (uint64_t)(n * C + j % C);
        const uint4 w = philox(i >> 3, offset, s.key0, s.key1);
        const uint64_t b = __ballot(number(w, (int)(i & 7)) < limit);
        if ((threadIdx.x & 63) == 0) bits[j >> 6] = b;
    }
    __syncthreads();
    const uint8_t* byte = (const uint8_t*)bits;
    // groups of eight values of the whole tensor that touch the sample, from the one that holds its first value on
    const long long first = n * voxels * C, last = first + voxels * C;
    const long long step = (long long)gridDim.x * 256;
    long long g = first / 8 + (long long)blockIdx.x * 256 + threadIdx.x;
    int c = (int)((8 * g - first + C * 8ll) % C);      // channel of the group's first value (the first group may begin up to 7 before)
    const int move = (int)(step * 8 % C);
    for (; 8 * g < last; g += step) {
        const uint32_t m = ((uint32_t)byte[c >> 3] | (uint32_t)byte[(c >> 3) + 1] << 8) >> (c & 7);
        if (8 * g >= first && 8 * g + 8 <= last) {
            float v[8];
            load_values<T, 8>(a + 8 * g, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = m >> j & 1 ? v[j] * scale : 0.f;
            store_values<T, 8>(out + 8 * g, v);
        } else {
            for (int j = 0; j < 8; ++j) {
                const long long i = 8 * g + j;
                if (i < first || i >= last) continue;
                float v[1];
                load_values<T, 1>(a + i, v);
                v[0] = m >> j & 1 ? v[0] * scale : 0.f;
                store_values<T, 1>(out + i, v);
            }
        }
        c += move;
        if (c >= C) c -= C;
    }
}

struct Kept {
    uint32_t limit;
    float scale;
};
bool kept_of(float p, Kept* k) {
    if (!(p >= 0.f && p <= 1.f)) return false;
    k->limit = (uint32_t)std::lround((1.0 - (double)p) * 65536.0);
    k->scale = k->limit ? (float)(65536.0 / k->limit) : 0.f;
    return true;
}
constexpr long long MOST_BLOCKS = 2048;

template <typename T>
int dropout(const void* a, const void* res, void* out, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t* more, void* stream) {
    Kept k;
    if (!kept_of(p, &k) || ((uintptr_t)more & 7) || !aligned16(a) || !aligned16(res) || !aligned16(out)) return MI3D_ERR_INVALID_ARG;
    if (n == 0) return MI3D_OK;
    if (!a || !out) return MI3D_ERR_INVALID_ARG;
    if (n >= (1ull << 50)) return MI3D_ERR_UNSUPPORTED;
    const Stream s = {(uint32_t)seed, (uint32_t)(seed >> 32), offset, more};
    const long long blocks = ((long long)n + 2047) / 2048;
    const unsigned grid = (unsigned)(blocks < MOST_BLOCKS ? blocks : MOST_BLOCKS);
    if (res) dropout_kernel<T, true><<<grid, 256, 0, (hipStream_t)stream>>>((const T*)a, (const T*)res, (T*)out, (long long)n, s, k.limit, k.scale);
    else dropout_kernel<T, false><<<grid, 256, 0, (hipStream_t)stream>>>((const T*)a, nullptr, (T*)out, (long long)n, s, k.limit, k.scale);
    return check_launch();
}

template <typename T>
int dropout_channels(const void* a, void* out, int N, size_t voxels, int C, float p, uint64_t seed, uint64_t offset, const uint64_t* more, void* stream) {
    Kept k;
    if (!kept_of(p, &k) || N < 0 || C <= 0 || ((uintptr_t)more & 7) || !aligned16(a) || !aligned16(out)) return MI3D_ERR_INVALID_ARG;
    if (N == 0 || voxels == 0) return MI3D_OK;
    if (!a || !out) return MI3D_ERR_INVALID_ARG;
    if (C > 65536 || N > 65535 || voxels >= (1ull << 30)) return MI3D_ERR_UNSUPPORTED;
    const Stream s = {(uint32_t)seed, (uint32_t)(seed >> 32), offset, more};
    const long long blocks = ((long long)voxels * C + 7 + 2047) / 2048, most = (MOST_BLOCKS + N - 1) / N;
    const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)N);
    dropout_channels_kernel<T><<<grid, 256, (size_t)(C + 16 + 255) / 256 * 32, (hipStream_t)stream>>>((const T*)a, (T*)out, (long long)voxels, C, s, k.limit, k.scale);
    return check_launch();
}

}  // namespace
}  // namespace mi3d

using namespace mi3d;

extern "C" {

int mi3d_dropout_fwd(const void* a, const void* residual, void* out, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout<uint16_t>(a, residual, out, n, p, seed, offset, dev_offset, stream);
}
int mi3d_dropout_fwd_f32(const float* a, const float* residual, float* out, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout<float>(a, residual, out, n, p, seed, offset, dev_offset, stream);
}
int mi3d_dropout_bwd(const void* dout, void* da, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout<uint16_t>(dout, nullptr, da, n, p, seed, offset, dev_offset, stream);
}
int mi3d_dropout_bwd_f32(const float* dout, float* da, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout<float>(dout, nullptr, da, n, p, seed, offset, dev_offset, stream);
}
int mi3d_dropout_channels(const void* a, void* out, int N, size_t voxels, int C, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout_channels<uint16_t>(a, out, N, voxels, C, p, seed, offset, dev_offset, stream);
}
int mi3d_dropout_channels_f32(const float* a, float* out, int N, size_t voxels, int C, float p, uint64_t seed, uint64_t offset, const uint64_t* dev_offset, void* stream) {
    return dropout_channels<float>(a, out, N, voxels, C, p, seed, offset, dev_offset, stream);
}

}  // extern "C"
