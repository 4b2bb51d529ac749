// Gated feed-forward block over the channels of each row (voxel or token).  With w1 = [gate; up] of F rows each:
//   [g | u] = x w1^T,  h = act(g) * u,  y = h w2^T                                                       (forward)
//   dh = dy w2,  dg = dh * u * act'(g),  du = dh * act(g),  h = act(g) * u,  dx = [dg | du] w1          (data gradient)
//   dw1 = [dg | du]^T x,  dw2 = dy^T h                                                                  (weight gradient, fp32)
//
// Every product is one kernel, D[m][n] = sum_k Q(m, k) P(n, k), whose operands lie in memory with k running along rows (x, w1, h,
// w2 in the forward pass) or across them (w2, w1 in the data gradient, everything in the weight gradient).  Each is fetched as it
// lies, by loads that go to LDS directly, 128 bytes of k a step: operands with k across are read from there transposed
// (bf16: ds_read_b64_tr_b16), so that no pass rewrites a tensor or the weights.  P goes into the first operand of the matrix
// instruction, whose results a lane then holds as four neighbouring n of one row.  bf16: v_mfma_f32_32x32x16_bf16; fp32:
// v_mfma_f32_32x32x2_f32 on the same 16-byte pieces, four of k.  Sums in fp32.  Bound: the matrix instructions.
#include <cmath>

#include "ig_common.h"
#include "mi3d_internal.h"
#include "rows_common.h"

namespace mi3d {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((address_space(3))) char* lds_char;
constexpr unsigned OOB = 0xFFFFFFF0u;      // buffer offset of a piece that must read as zero

// What happens to the results.  GATE: P holds gate and up rows in turn, h (and g, u) come out.  DACT: the results are dh.
// PART: fp32 results, or the sums of a part of the contraction.
enum Form { STORE, GATE, DACT, PART };

struct FfnParams {
    const void *q, *p;
    long long M, K;
    int N, qp, pp;             // columns of D; elements from one row of Q's and P's memory to the next
    int F, act;
    void *out, *out2;          // STORE, PART: D.  GATE: h, [g | u] or null.  DACT: h, [dg | du]
    const void* gu;            // DACT
    int mt, nt, splits;
    long long steps;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const char* p, long long bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes > 0x7fffffffll ? 0x7fffffff : bytes < 0 ? 0 : (int)bytes, 0x00020000);
}

// act(g) and act'(g); silu: g s(g) with the logistic s, gelu: g Phi(g) with the normal distribution's Phi
__device__ __forceinline__ float activation(float g, int act) {
    if (act == MI3D_ACT_SILU) return g / (1.f + expf(-g));
    return 0.5f * g * (1.f + erff(g * 0.70710678f));
}
__device__ __forceinline__ void activation(float g, int act, float& a, float& d) {
    if (act == MI3D_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-g));
        a = g * s;
        d = s * (1.f + g * (1.f - s));
    } else {
        const float c = 0.5f * (1.f + erff(g * 0.70710678f));
        a = g * c;
        d = c + g * 0.39894228f * expf(-0.5f * g * g);
    }
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&f)[4]) {
    if constexpr (sizeof(T) == 2) {
        const uint2 v = *(const uint2*)p;
        f[0] = __builtin_bit_cast(float, v.x << 16);
        f[1] = __builtin_bit_cast(float, v.x & 0xFFFF0000u);
        f[2] = __builtin_bit_cast(float, v.y << 16);
        f[3] = __builtin_bit_cast(float, v.y & 0xFFFF0000u);
    } else {
        const float4 v = *(const float4*)p;
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&f)[4]) {
    if constexpr (sizeof(T) == 2) *(uint2*)p = uint2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
    else *(float4*)p = float4{f[0], f[1], f[2], f[3]};
}

// One operand's share of a step in LDS: R rows of 128 bytes of k (ACROSS false), or 128 / sizeof(T) rows of k of R values.  16-byte
// pieces are permuted inside a row so that the lanes of a read fall into different banks.
template <typename T, int R, bool ACROSS>
struct Operand {
    static constexpr int E = sizeof(T), KS = 128 / E, ROW = ACROSS ? R * E : 128, PER = ROW / 16;    // bytes, pieces of a row
    static __device__ __forceinline__ int swizzle(int row) {
        if (!ACROSS) return row & 7;
        if (E == 4) return 2 * (row & 4);
        return ROW >= 256 ? 4 * (row & 3) : 2 * (row & 2);
    }
    // fragments of the block of 32 that begins at `at`, of the kk-th sixteen (fp32: eight) k of the step
    static __device__ __forceinline__ int place(int at, int lane) {
        const int ln = lane & 31, half = lane >> 5;
        if (!ACROSS) return (at + ln) * 128;      // (the piece depends on kk)
        if (E == 4) return 4 * half * ROW + ((((at + ln) >> 2) ^ (8 * half)) << 4) + (ln & 3) * 4;
        const int g = lane >> 4, row = 8 * (g >> 1) + (lane >> 2 & 3), c8 = lane & 3;
        return row * ROW + ((((at + 16 * (g & 1)) / 8 + (c8 >> 1)) ^ swizzle(row)) << 4) + (c8 & 1) * 8;
    }
    struct Frag {
        bf16x8 h;
        float f[4];
    };
    static __device__ __forceinline__ Frag read(const char* l, int place, int kk, int lane) {
        Frag r;
        if constexpr (!ACROSS) {
            const char* p = l + place + (((2 * kk + (lane >> 5)) ^ (lane & 7)) << 4);      // (blocks begin at multiples of 32)
            if constexpr (E == 2) r.h = *(const bf16x8*)p;
            else {
                const float4 v = *(const float4*)p;
                r.f[0] = v.x; r.f[1] = v.y; r.f[2] = v.z; r.f[3] = v.w;
            }
        } else if constexpr (E == 2) {
            r.h = tr_frag(l + place + kk * 16 * ROW, ROW);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) r.f[j] = *(const float*)(l + place + (8 * kk + j) * ROW);
        }
        return r;
    }
};

// A workgroup of WM x WN waves owns 32 MB WM rows x 64 WN columns of D (GATE: columns of g and of u, half each); a wave MB x 2 blocks of
// 32 x 32.  Two stages of LDS: a step's loads run while the step before is computed.
template <typename T, int MB, int WM, int WN, bool QA, bool PA, Form FORM>
__global__ void __launch_bounds__(64 * WM * WN, 2) ffn_gemm_kernel(const FfnParams P) {
    constexpr int W = WM * WN, BM = 32 * MB * WM, BN = 64 * WN, E = sizeof(T), KS = 128 / E;
    constexpr int NQ = BM / (8 * W), NP = BN / (8 * W), Q_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    typedef Operand<T, BM, QA> OQ;
    typedef Operand<T, BN, PA> OP;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);

    // block -> (part, tile); the blocks of an XCD (every eighth) get neighbouring tiles, four tiles of rows by all of columns at a time
    const int tiles = P.mt * P.nt;
    int id;
    {
        const int n = tiles * P.splits, l = blockIdx.x, x = l & 7, q = l >> 3;
        id = x * (n >> 3) + ((n & 7) < x ? (n & 7) : x) + q;
    }
    const int split = id / tiles;
    id -= split * tiles;
    const int band = id / (4 * P.nt), in = id - band * 4 * P.nt, high = P.mt - 4 * band < 4 ? P.mt - 4 * band : 4;
    const int mt = 4 * band + in % high, nt = in / high;
    const long long s0 = P.steps * split / P.splits, s1 = P.steps * (split + 1) / P.splits;

    const long long m0 = (long long)mt * BM, kbytes = P.K * E;
    const int n0 = nt * (FORM == GATE ? BN / 2 : BN);
    const long long qrow = (long long)P.qp * E, prow = (long long)P.pp * E;
    // byte offsets of the pieces this lane fetches in the buffers below
    unsigned qo[NQ], po[NP];
    const int kq = ((lane & 7) ^ (lane >> 3)) * 16;      // (k along: byte of k inside a step)
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int g = i * W + wave;
        if constexpr (QA) {
            const int row = g * 64 / OQ::PER + lane / OQ::PER;
            qo[i] = (unsigned)(row * qrow + ((lane % OQ::PER) ^ OQ::swizzle(row)) * 16);
        } else qo[i] = (unsigned)((8 * g + (lane >> 3)) * qrow + kq);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int g = i * W + wave;
        if constexpr (PA) {
            const int row = g * 64 / OP::PER + lane / OP::PER;
            po[i] = (unsigned)(row * prow + ((lane % OP::PER) ^ OP::swizzle(row)) * 16);
        } else {
            // GATE: 32 rows of the gate, the same 32 of up, ...
            const int row = FORM == GATE ? 32 * (g >> 3) + 8 * (g & 3) : 8 * g;
            po[i] = (unsigned)((row + (lane >> 3)) * prow + kq);
        }
    }
    const unsigned lds_wave = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char)lds) + wave * 1024;
    const char *q = (const char*)P.q, *p = (const char*)P.p;
    auto fetch = [&](long long s) {
        const unsigned l = lds_wave + (unsigned)((s - s0) & 1) * STAGE;
        const long long k = s * 128;                     // (k along) byte of k
        {
            const long long at = QA ? s * KS * qrow + m0 * E : m0 * qrow;
            const __amdgpu_buffer_rsrc_t r = buffer(q + at, (QA ? P.K : P.M) * qrow - at);
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                load_lds_asm(r, l + i * W * 1024, QA ? qo[i] : k + kq < kbytes ? qo[i] + (unsigned)k : OOB);
        }
        const long long at = PA ? s * KS * prow + (long long)n0 * E : n0 * prow;
        const long long all = PA ? P.K * prow : (FORM == GATE ? P.F : P.N) * prow;
        const __amdgpu_buffer_rsrc_t r = buffer(p + at, all - at);
        const __amdgpu_buffer_rsrc_t r2 = buffer(p + at + (FORM == GATE ? all : 0), all - at);
#pragma unroll
        for (int i = 0; i < NP; ++i)
            load_lds_asm(FORM == GATE && (i * W + wave) & 4 ? r2 : r, l + Q_BYTES + i * W * 1024, PA ? po[i] : k + kq < kbytes ? po[i] + (unsigned)k : OOB);
    };

    f32x16 acc[MB][2];
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

    const int wm = (wave % WM) * 32 * MB, wn = (wave / WM) * 64;
    int fq[MB], fp[2];
#pragma unroll
    for (int a = 0; a < MB; ++a) fq[a] = OQ::place(wm + 32 * a, lane);
#pragma unroll
    for (int b = 0; b < 2; ++b) fp[b] = Q_BYTES + OP::place(wn + 32 * b, lane);

    if (s0 < s1) fetch(s0);
    for (long long s = s0; s < s1; ++s) {
        // this step's pieces have come, in all waves, and all have read the step before
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < s1) fetch(s + 1);
        const char* l = lds + ((s - s0) & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            typename OQ::Frag vq[MB];
            typename OP::Frag vp[2];
#pragma unroll
            for (int a = 0; a < MB; ++a) vq[a] = OQ::read(l, fq[a], kk, lane);
#pragma unroll
            for (int b = 0; b < 2; ++b) vp[b] = OP::read(l, fp[b], kk, lane);
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    if constexpr (E == 2) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[b].h, vq[a].h, acc[a][b], 0, 0, 0);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[b].f[j], vq[a].f[j], acc[a][b], 0, 0, 0);
                }
        }
    }

    // lane (row ln, half): registers 4 i .. 4 i + 3 of a block are columns 8 i + 4 half .. + 3 of its 32
    const int ln = lane & 31, half = lane >> 5;
#pragma unroll
    for (int a = 0; a < MB; ++a) {
        const long long m = m0 + wm + 32 * a + ln;
        if (m >= P.M) continue;
        if constexpr (FORM == GATE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f = n0 + wn / 2 + 8 * i + 4 * half;
                if (f >= P.F) continue;
                float g[4], u[4], h[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    g[j] = acc[a][0][4 * i + j];
                    u[j] = acc[a][1][4 * i + j];
                    h[j] = activation(g[j], P.act) * u[j];      // (of the sums, not of what is kept of them)
                }
                store4((T*)P.out + m * P.F + f, h);
                if (P.out2) {
                    store4((T*)P.out2 + m * 2 * P.F + f, g);
                    store4((T*)P.out2 + m * 2 * P.F + P.F + f, u);
                }
            }
        } else {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = n0 + wn + 32 * b + 8 * i + 4 * half;
                    if (n >= P.N) continue;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[a][b][4 * i + j];
                    if constexpr (FORM == STORE) store4((T*)P.out + m * P.N + n, v);
                    if constexpr (FORM == PART) store4((float*)P.out + ((long long)split * P.M + m) * P.N + n, v);
                    if constexpr (FORM == DACT) {
                        float g[4], u[4], h[4];
                        load4((const T*)P.gu + m * 2 * P.N + n, g);
                        load4((const T*)P.gu + m * 2 * P.N + P.N + n, u);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float c, d;
                            activation(g[j], P.act, c, d);
                            h[j] = c * u[j];
                            g[j] = v[j] * u[j] * d;
                            u[j] = v[j] * c;
                        }
                        store4((T*)P.out + m * P.N + n, h);
                        store4((T*)P.out2 + m * 2 * P.N + n, g);
                        store4((T*)P.out2 + m * 2 * P.N + P.N + n, u);
                    }
                }
        }
    }
}

long long tiles_of(long long n, int tile) { return (n + tile - 1) / tile; }

template <typename T, bool QA, bool PA, Form FORM>
int gemm(FfnParams P, hipStream_t s) {
    constexpr int MB = 2, WM = 2, WN = 2, BM = 32 * MB * WM, BN = 64 * WN, STAGES = 2 * (BM + BN) * 128;
    P.mt = (int)tiles_of(P.M, BM);
    P.nt = (int)tiles_of(FORM == GATE ? P.F : P.N, FORM == GATE ? BN / 2 : BN);
    P.steps = tiles_of(P.K, 128 / sizeof(T));
    if (P.splits < 1) P.splits = 1;
    const auto kernel = ffn_gemm_kernel<T, MB, WM, WN, QA, PA, FORM>;
    const long long grid = (long long)P.mt * P.nt * P.splits;
    if (grid == 0) return MI3D_OK;
    if (grid >= (1ll << 31)) return MI3D_ERR_UNSUPPORTED;
    static std::atomic<bool> attr_set{false};   // set once per process; a second thread racing here repeats an idempotent call
    if (!attr_set) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, STAGES);
        if (e != hipSuccess) { note_hip_error(e); return MI3D_ERR_HIP; }
        attr_set = true;
    }
    kernel<<<(unsigned)grid, 64 * WM * WN, STAGES, s>>>(P);
    return check_launch();
}

// parts of the contraction of a weight gradient, so that its tiles fill the chip
int wgrad_splits(long long M, long long N, long long K, int e) {
    const long long tiles = tiles_of(M, 128) * tiles_of(N, 128), steps = tiles_of(K, 128 / e);
    long long s = 2 * 256 / tiles;
    if (s > steps / 4) s = steps / 4;
    return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

struct Desc {
    long long rows;
    int C, F, O, act, e;
};
int make(const mi3d_ffn_desc* d, Desc* o) {
    if (!d || d->rows < 0 || d->Cin <= 0 || d->F <= 0 || d->Cout <= 0) return MI3D_ERR_INVALID_ARG;
    if (d->act != MI3D_ACT_SILU && d->act != MI3D_ACT_GELU) return MI3D_ERR_UNSUPPORTED;
    if (d->dtype != MI3D_F32 && d->dtype != MI3D_BF16) return MI3D_ERR_UNSUPPORTED;
    if (d->Cin % 8 || d->F % 8 || d->Cout % 8) return MI3D_ERR_UNSUPPORTED;
    if (d->rows >= (1ll << 31) || d->Cin > 65536 || d->F > 65536 || d->Cout > 65536) return MI3D_ERR_UNSUPPORTED;
    *o = Desc{d->rows, d->Cin, d->F, d->Cout, d->act, d->dtype == MI3D_BF16 ? 2 : 4};
    return MI3D_OK;
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t workspace(const Desc& d, int pass) {
    if (pass == MI3D_PASS_FWD) return round256((size_t)d.rows * d.F * d.e);      // h
    if (pass != MI3D_PASS_WGRAD) return 0;
    const int s1 = wgrad_splits(2 * d.F, d.C, d.rows, d.e), s2 = wgrad_splits(d.O, d.F, d.rows, d.e);
    const size_t n1 = s1 > 1 ? (size_t)s1 * 2 * d.F * d.C * 4 : 0, n2 = s2 > 1 ? (size_t)s2 * d.O * d.F * 4 : 0;
    return n1 > n2 ? n1 : n2;
}
bool usable(const void* p) { return p && aligned16(p); }

template <typename T>
int gate(const Desc& d, const void* x, const void* w1, void* h, void* gu, hipStream_t s) {
    FfnParams P{};
    P.q = x; P.p = w1; P.M = d.rows; P.K = d.C; P.N = d.F; P.qp = d.C; P.pp = d.C; P.F = d.F; P.act = d.act;
    P.out = h; P.out2 = gu;
    return gemm<T, false, false, GATE>(P, s);
}
template <typename T>
int project(const Desc& d, const void* h, const void* w2, void* y, hipStream_t s) {
    FfnParams P{};
    P.q = h; P.p = w2; P.M = d.rows; P.K = d.F; P.N = d.O; P.qp = d.F; P.pp = d.F; P.out = y;
    return gemm<T, false, false, STORE>(P, s);
}
template <typename T>
int dgrad(const Desc& d, const void* dy, const void* w1, const void* w2, const void* gu, void* dgu, void* h, void* dx, hipStream_t s) {
    FfnParams P{};
    P.q = dy; P.p = w2; P.M = d.rows; P.K = d.O; P.N = d.F; P.qp = d.O; P.pp = d.F; P.act = d.act;
    P.out = h; P.out2 = dgu; P.gu = gu;
    const int st = gemm<T, false, true, DACT>(P, s);
    if (st) return st;
    FfnParams R{};
    R.q = dgu; R.p = w1; R.M = d.rows; R.K = 2 * d.F; R.N = d.C; R.qp = 2 * d.F; R.pp = d.C; R.out = dx;
    return gemm<T, false, true, STORE>(R, s);
}
// out[m][n] = sum over rows of a[row][m] b[row][n]
template <typename T>
int outer(const void* a, const void* b, long long rows, int M, int N, float* out, void* ws, hipStream_t s) {
    FfnParams P{};
    P.q = a; P.p = b; P.M = M; P.K = rows; P.N = N; P.qp = M; P.pp = N;
    P.splits = wgrad_splits(M, N, rows, sizeof(T));
    P.out = P.splits > 1 ? ws : out;
    const int st = gemm<T, true, true, PART>(P, s);
    return st || P.splits == 1 ? st : reduce_partials((const float*)ws, out, (long long)M * N, P.splits, s);
}

}  // namespace
}  // namespace mi3d

using namespace mi3d;

extern "C" {

size_t mi3d_ffn_workspace_bytes(const mi3d_ffn_desc* desc, int pass) {
    Desc d;
    return make(desc, &d) == MI3D_OK ? workspace(d, pass) : 0;
}

int mi3d_ffn_gate(const mi3d_ffn_desc* desc, const void* x, const void* w1, void* h, void* gu, void* stream) {
    Desc d;
    const int st = make(desc, &d);
    if (st) return st;
    if (!usable(w1) || !aligned16(x) || !aligned16(h) || !aligned16(gu)) return MI3D_ERR_INVALID_ARG;
    if (d.rows == 0) return MI3D_OK;
    if (!x || !h) return MI3D_ERR_INVALID_ARG;
    return d.e == 2 ? gate<uint16_t>(d, x, w1, h, gu, (hipStream_t)stream) : gate<float>(d, x, w1, h, gu, (hipStream_t)stream);
}

int mi3d_ffn_fwd(const mi3d_ffn_desc* desc, const void* x, const void* w1, const void* w2, void* y, void* gu, void* ws, size_t ws_bytes, void* stream) {
    Desc d;
    int st = make(desc, &d);
    if (st) return st;
    if (!usable(w1) || !usable(w2) || !aligned16(x) || !aligned16(y) || !aligned16(gu) || !aligned16(ws)) return MI3D_ERR_INVALID_ARG;
    if (d.rows == 0) return MI3D_OK;
    if (!x || !y) return MI3D_ERR_INVALID_ARG;
    if (!ws || ws_bytes < workspace(d, MI3D_PASS_FWD)) return MI3D_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    st = d.e == 2 ? gate<uint16_t>(d, x, w1, ws, gu, s) : gate<float>(d, x, w1, ws, gu, s);
    if (st) return st;
    return d.e == 2 ? project<uint16_t>(d, ws, w2, y, s) : project<float>(d, ws, w2, y, s);
}

int mi3d_ffn_dgrad(const mi3d_ffn_desc* desc, const void* dy, const void* w1, const void* w2, const void* gu, void* dgu, void* h, void* dx,
                   void* ws, size_t ws_bytes, void* stream) {
    Desc d;
    const int st = make(desc, &d);
    if (st) return st;
    if (!usable(w1) || !usable(w2) || !aligned16(dy) || !aligned16(gu) || !aligned16(dgu) || !aligned16(h) || !aligned16(dx) || !aligned16(ws))
        return MI3D_ERR_INVALID_ARG;
    if (d.rows == 0) return MI3D_OK;
    if (!dy || !gu || !dgu || !h || !dx) return MI3D_ERR_INVALID_ARG;
    const size_t need = workspace(d, MI3D_PASS_DGRAD);
    if (need && (!ws || ws_bytes < need)) return MI3D_ERR_WORKSPACE;
    return d.e == 2 ? dgrad<uint16_t>(d, dy, w1, w2, gu, dgu, h, dx, (hipStream_t)stream) : dgrad<float>(d, dy, w1, w2, gu, dgu, h, dx, (hipStream_t)stream);
}

int mi3d_ffn_wgrad(const mi3d_ffn_desc* desc, const void* x, const void* dgu, const void* h, const void* dy, float* dw1, float* dw2,
                   void* ws, size_t ws_bytes, void* stream) {
    Desc d;
    int st = make(desc, &d);
    if (st) return st;
    if (!usable(dw1) || !usable(dw2) || !aligned16(x) || !aligned16(dgu) || !aligned16(h) || !aligned16(dy) || !aligned16(ws)) return MI3D_ERR_INVALID_ARG;
    if (d.rows && (!x || !dgu || !h || !dy)) return MI3D_ERR_INVALID_ARG;
    const size_t need = workspace(d, MI3D_PASS_WGRAD);
    if (need && (!ws || ws_bytes < need)) return MI3D_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    st = d.e == 2 ? outer<uint16_t>(dgu, x, d.rows, 2 * d.F, d.C, dw1, ws, s) : outer<float>(dgu, x, d.rows, 2 * d.F, d.C, dw1, ws, s);
    if (st) return st;
    return d.e == 2 ? outer<uint16_t>(dy, h, d.rows, d.O, d.F, dw2, ws, s) : outer<float>(dy, h, d.rows, d.O, d.F, dw2, ws, s);
}

}  // extern "C"
