// Gated feed-forward block over the channels of each row (voxel or token).  With w1 = [gate; up] of F rows each:
//   [g | u] = x w1^T,  h = act(g) * u,  y = h w2^T                                                       (forward)
//   dh = dy w2,  dg = dh * u * act'(g),  du = dh * act(g),  h = act(g) * u,  dx = [dg | du] w1          (data gradient)
//   dw1 = [dg | du]^T x,  dw2 = dy^T h                                                                  (weight gradient, fp32)
//
// Every product is one kernel, D[m][n] = sum_k Q(m, k) P(n, k), whose operands lie in memory with k running along rows (x, w1, h,
// w2 in the forward pass) or across them (w2, w1 in the data gradient, everything in the weight gradient).  Each is fetched as it
// lies, by loads that go to LDS directly, 64 or 128 bytes of k a step: operands with k across are read from there transposed
// (bf16: ds_read_b64_tr_b16), so that no pass rewrites a tensor or the weights.  P goes into the first operand of the matrix
// instruction, whose results a lane then holds as four neighbouring n of one row.  bf16: v_mfma_f32_32x32x16_bf16; fp32:
// v_mfma_f32_32x32x2_f32 on the same 16-byte pieces, four of k.  Sums in fp32.
//
// Rounded to the type on the way, beside the results themselves: h between the two forward products, and [dg | du] before dx is formed
// from it (dx thus belongs to the [dg | du] that the weight gradient reads).  In bf16 both are operands of instructions that take
// bf16; in two parts each they would double their product's k, 42 -> 72 us of 131 (forward, 27648 x 320 x 1280) and 237 -> 462 of 483
// (data gradient, 16384 x 1024 x 4096).  What it costs: an error against 64 bits of 2.3e-3 to 2.4e-3 in the 2-norm, where one rounding at
// the end has 1.65e-3.  h and the activation's derivative in the data gradient come from the rounded [g | u], the only one that is
// kept, so dw2 reads an h that is up to a rounding of g and u off the forward pass's.  Whoever needs more takes fp32.
//
// Bound: the matrix instructions on long contractions (dx of 8192 x 4096 x 8192: 913 us, 1204 TFLOP/s, where a library product of 8192^3
// reaches 1294; fp32, 16384 x 1024 x 4096: 134 to 139, and 131, the data gradient's first product 120); the results of short ones, which
// every workgroup has to write (and for the data gradient read [g | u]) before its compute unit goes on: 16384 x 1024 x 4096 data gradient
// 247 + 237 us, 27648 x 320 x 1280 forward 89 + 42 us (three sets of tensors in turn; 228 + 227 and 75 + 43 on one set again and again).
// Measured on the way (16384 x 1024 x 4096, data gradient): results straight from registers, 8 bytes a lane, 811 us; through LDS 571;
// without bank conflicts the same; fragments a turn ahead and loads between the products 475; results streamed 10 less (below).  Not
// faster: two to four workgroups of smaller tiles on a unit, deeper rings, workgroups of a unit out of step, wave priorities.

#include <cstdio>

#include "ffn.h"
#include "ig_common.h"

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
    int F;
    void *out, *out2;          // STORE, PART: D.  GATE: h, [g | u] or null.  DACT: h, [dg | du]
    const void* gu;            // DACT
    int splits, per, extra;    // parts of the contraction; steps of a part, one more of the first `extra`
    Div tiles, band, last;     // of a part, of four tiles of rows (`last`: of rows in the last such band)
    int mt, nt;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const char* p, long long bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes > 0x7fffffffll ? 0x7fffffff : bytes < 0 ? 0 : (int)bytes, 0x00020000);
}

// eight values as they lie in memory
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
template <typename T>
struct Eight {
    u32x4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load_streamed(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) v[i] = __builtin_nontemporal_load((const u32x4*)p + i);
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const { load_values<T, 8>((const T*)v, f); }
};

// One operand's share of a step in LDS: R rows of KB bytes of k (ACROSS false), or KB / sizeof(T) rows of k of R values.  16-byte
// pieces are permuted inside a row so that the lanes of a read fall into different banks.
template <typename T, int R, int KB, bool ACROSS>
struct Operand {
    static constexpr int E = sizeof(T), ROW = ACROSS ? R * E : KB, PER = ROW / 16;    // bytes, pieces of a row
    static __device__ __forceinline__ int swizzle(int row) {
        if (!ACROSS) return KB == 128 ? row >> 1 & 7 : row >> 2 & 3;      // (sixteen rows fill the 256 bytes of the banks)
        if (E == 4) return 2 * (row & 4);
        return ROW >= 256 ? 4 * (row & 3) : 2 * (row & 2);
    }
    // fragments of the block of 32 that begins at `at` (a multiple of 32)
    static __device__ __forceinline__ int place(int at, int lane) {
        const int ln = lane & 31, half = lane >> 5;
        if (!ACROSS) return (at + ln) * KB;      // (the piece depends on kk)
        if (E == 4) return 4 * half * ROW + ((((at + ln) >> 2) ^ (8 * half)) << 4) + (ln & 3) * 4;
        const int g = lane >> 4, row = 8 * (g >> 1) + (lane >> 2 & 3), c8 = lane & 3;
        return row * ROW + ((((at + 16 * (g & 1)) / 8 + (c8 >> 1)) ^ swizzle(row)) << 4) + (c8 & 1) * 8;
    }
    struct Frag {
        bf16x8 h;
        float f[4];
    };
    // of the kk-th sixteen (fp32: eight) k of the step
    static __device__ __forceinline__ Frag read(const char* l, int place, int kk, int lane) {
        Frag r;
        if constexpr (!ACROSS) {
            const char* p = l + place + (((2 * kk + (lane >> 5)) ^ swizzle(lane & 31)) << 4);
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
// 32 x 32.  A step is KB bytes of k; RING steps have a place in LDS, of which RING - 1 come in while one is computed.
template <typename T, int MB, int WM, int WN, int KB, int RING, bool QA, bool PA, Form FORM, int ACT>
__device__ __forceinline__ void ffn_tile(const FfnParams& P, const int block) {
    constexpr int W = WM * WN, BM = 32 * MB * WM, BN = 64 * WN, E = sizeof(T), KS = KB / E;
    constexpr int NQ = BM * KB / 1024 / W, NP = BN * KB / 1024 / W, Q_BYTES = BM * KB, STAGE = (BM + BN) * KB;
    constexpr int ROWS = 1024 / KB;      // (k along) rows of a wave's load
    typedef Operand<T, BM, KB, QA> OQ;
    typedef Operand<T, BN, KB, PA> OP;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);

    // block -> (part, tile); the blocks of an XCD (every eighth) get neighbouring tiles, four tiles of rows by all of columns at a time
    int id;
    {
        const int n = (int)P.tiles.d * P.splits, l = block, x = l & 7, q = l >> 3;
        id = x * (n >> 3) + ((n & 7) < x ? (n & 7) : x) + q;
    }
    const int split = divide(id, P.tiles);
    id -= split * (int)P.tiles.d;
    const int band = divide(id, P.band), in = id - band * (int)P.band.d;
    const bool whole = 4 * band + 4 <= P.mt;
    const int nt = whole ? in >> 2 : divide(in, P.last), mt = 4 * band + (whole ? in & 3 : in - nt * (int)P.last.d);
    const int s0 = split * P.per + (split < P.extra ? split : P.extra), s1 = s0 + P.per + (split < P.extra ? 1 : 0);

    const long long m0 = (long long)mt * BM, kbytes = P.K * E;
    const int n0 = nt * (FORM == GATE ? BN / 2 : BN);
    const long long qrow = (long long)P.qp * E, prow = (long long)P.pp * E;
    // byte offsets of the pieces this lane fetches in the buffers below
    unsigned qo[NQ], po[NP];
    const int rl = lane / (KB / 16), kq = ((lane % (KB / 16)) ^ Operand<T, BM, KB, false>::swizzle(ROWS * (wave & 1) + rl)) * 16;      // (k along) row of the load, byte of k inside a step
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int g = i * W + wave;
        if constexpr (QA) {
            const int row = g * 64 / OQ::PER + lane / OQ::PER;
            qo[i] = (unsigned)(row * qrow + ((lane % OQ::PER) ^ OQ::swizzle(row)) * 16);
        } else qo[i] = (unsigned)((ROWS * g + rl) * qrow + kq);
    }
    auto up = [&](int i) { return FORM == GATE && (ROWS * (i * W + wave) & 32); };      // GATE: 32 rows of the gate, the same 32 of up, ...
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int g = i * W + wave;
        if constexpr (PA) {
            const int row = g * 64 / OP::PER + lane / OP::PER;
            po[i] = (unsigned)(row * prow + ((lane % OP::PER) ^ OP::swizzle(row)) * 16);
        } else {
            const int row = FORM == GATE ? 32 * (ROWS * g / 64) + ROWS * g % 32 : ROWS * g;
            po[i] = (unsigned)((row + rl) * prow + kq);
        }
    }
    const unsigned lds_wave = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char)lds) + wave * 1024;
    const char *q = (const char*)P.q, *p = (const char*)P.p;
    // The step under way to LDS: its place and buffers (of no bytes behind the last step: loads that write zeros where nobody reads)
    unsigned slot_in = 0, to = 0;
    bool inside = false;                                 // (k along) this lane's piece lies before the end of k
    __amdgpu_buffer_rsrc_t rq = buffer(q, 0), rp = rq, ru = rq;
    auto begin = [&](int s) {
        to = lds_wave + slot_in * STAGE;
        slot_in = slot_in + 1 == RING ? 0 : slot_in + 1;
        const long long k = (long long)s * KB, none = s < s1 ? 0 : 1ll << 62;
        inside = k + kq < kbytes;
        const long long aq = QA ? (long long)s * KS * qrow + m0 * E : m0 * qrow + k;
        rq = buffer(q + aq, (QA ? P.K : P.M) * qrow - aq - none);
        const long long ap = PA ? (long long)s * KS * prow + (long long)n0 * E : n0 * prow + k;
        const long long all = PA ? P.K * prow : (FORM == GATE ? P.F : P.N) * prow;
        rp = buffer(p + ap, all - ap - none);
        if (FORM == GATE) ru = buffer(p + ap + all, all - ap - none);
    };
    constexpr int NL = NQ + NP;
    auto load = [&](int i) {
        if (i < NQ) load_lds_asm(rq, to + i * W * 1024, QA || inside ? qo[i] : OOB);
        else load_lds_asm(up(i - NQ) ? ru : rp, to + Q_BYTES + (i - NQ) * W * 1024, PA || inside ? po[i - NQ] : OOB);
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

    // A step is KK turns of sixteen (fp32: eight) k.  Between a turn's products stand the reads of the next turn's fragments and a
    // share of a step's loads, so that no wave stands in line for LDS or the address unit while its matrix unit idles; before the last
    // turn's stands the barrier behind which the next step is read and this step's place filled.
    constexpr int KK = KB / 32, NR = MB + 2, NM = 2 * MB, TP = 2;      // TP: turns that share a step's loads (1 and 4: up to 7 % slower)
    typename OQ::Frag vq[2][MB];
    typename OP::Frag vp[2][2];
    auto read = [&](const char* l, int kk, int to, int j) {      // in the order of the products
        if (j == 0 || j == 2) vp[to][j / 2] = OP::read(l, fp[j / 2], kk, lane);
        else vq[to][j == 1 ? 0 : j - 2] = OQ::read(l, fq[j == 1 ? 0 : j - 2], kk, lane);
    };
    if (s0 < s1) {
#pragma unroll
        for (int i = 0; i < RING; ++i) {
            begin(s0 + i);
#pragma unroll
            for (int j = 0; j < NL; ++j)
                if (i < RING - 1 || j < NL / TP) load(j);      // (the rest of the last one in the first step's turns)
        }
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((RING - 2) * NL + NL / TP) : "memory");
#pragma unroll
        for (int j = 0; j < NR; ++j) read(lds, 0, 0, j);
    }
    const char* l = lds;
    unsigned slot = 0;
    for (int s = s0; s < s1; ++s) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk == KK - 1) {
                // the next step's pieces have come (those of the RING - 2 behind it may be under way), in all waves, and all have read this step
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((RING - 2) * NL) : "memory");
                begin(s + RING);
                slot = slot + 1 == RING ? 0 : slot + 1;
                l = lds + slot * STAGE;
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int a = m / 2, b = m % 2;
                const typename OP::Frag& x = vp[kk & 1][b];
                const typename OQ::Frag& y = vq[kk & 1][a];
                if constexpr (E == 2) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.h, y.h, acc[a][b], 0, 0, 0);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.f[j], y.f[j], acc[a][b], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < NR; ++j)
                    if (j * NM / NR == m) read(l, kk < KK - 1 ? kk + 1 : 0, (kk + 1) & 1, j);
                const int part = kk == KK - 1 ? 0 : kk + 1;      // of the step's loads
                if (part < TP) {
                    const int j0 = NL * part / TP, j1 = NL * (part + 1) / TP;
#pragma unroll
                    for (int j = j0; j < j1; ++j)
                        if ((j - j0) * NM / (j1 - j0) == m) load(j);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the loads behind the last step)

    // (GATE, DACT: what comes and goes here is several times what the operands are, which stay in L2 if it is streamed past them: the two
    // products of 16384 x 1024 x 4096's data gradient 238 + 229 -> 228 + 227 us.  h, which the next product reads, goes past L2 as well: 27648 x
    // 320 x 1280 forward 76 + 40 -> 75 + 43.)
    // The results go through LDS (a lane holds four columns of one row; 16-byte pieces permuted by the row) so that each row's are
    // read and written in whole lines, eight values a thread, RA of the MB blocks of rows at a time.  The data gradient's g and u
    // are requested before.
    constexpr int BLOCKS = RING * STAGE / (32 * WM * BN * 4), RA = BLOCKS < MB ? BLOCKS : MB;
    static_assert(RA > 0 && MB % RA == 0, "");
    constexpr int SPREAD = BN / 4 < 32 ? BN / 4 - 1 : 31;
    constexpr int COLS = FORM == GATE ? BN / 2 : BN, PER = COLS / 8, TURNS = 32 * RA * WM * PER / (64 * W), MOST = 16 / E / 2, CH = FORM != DACT ? 1 : TURNS < MOST ? TURNS : MOST;
    static_assert(TURNS % CH == 0, "");
    const int width = FORM == GATE ? P.F : P.N;
    const int c8 = t % PER, n = n0 + 8 * c8;      // (64 W is a multiple of PER)
#pragma unroll
    for (int a0 = 0; a0 < MB; a0 += RA) {
    auto row_of = [&](int turn) {                 // of LDS
        return (turn * 64 * W + t) / PER;
    };
    auto m_of = [&](int row) { return m0 + row / (32 * RA) * (32 * MB) + 32 * a0 + row % (32 * RA); };
    Eight<T> g8[CH], u8[CH];
    auto request = [&](int turn) {
        if constexpr (FORM == DACT)
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const long long m = m_of(row_of(turn + i));
                if (m < P.M && n < width) {
                    const T* at = (const T*)P.gu + m * 2 * width + n;
                    g8[i].load_streamed(at);
                    u8[i].load_streamed(at + width);
                }
            }
    };
    request(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // all waves have read the last step, or the results before
    {
        const int ln = lane & 31, half = lane >> 5;
#pragma unroll
        for (int a = 0; a < RA; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x16& v = acc[a0 + a][b];
                    const int row = wave % WM * 32 * RA + 32 * a + ln, piece = (wn + 32 * b + 8 * i + 4 * half) / 4;
                    *(float4*)(lds + row * BN * 4 + ((piece ^ (ln & SPREAD)) << 4)) = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
                }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    auto take = [&](int row, int col, float (&v)[8]) {      // eight results, col a multiple of 8
        const char* l = lds + row * BN * 4;
        const float4 x = *(const float4*)(l + (((col / 4) ^ (row & SPREAD)) << 4)), y = *(const float4*)(l + (((col / 4 + 1) ^ (row & SPREAD)) << 4));
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    };
#pragma unroll
    for (int turn = 0; turn < TURNS; turn += CH) {
        float g[CH][8], u[CH][8];
        if constexpr (FORM == DACT) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                g8[i].unpack(g[i]);
                u8[i].unpack(u[i]);
            }
            if (turn + CH < TURNS) request(turn + CH);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int row = row_of(turn + i);
            const long long m = m_of(row);
            if (m >= P.M || n >= width) continue;
            float v[8];
            if constexpr (FORM == GATE) {
                take(row, (c8 >> 2) * 64 + (c8 & 3) * 8, g[0]);
                take(row, (c8 >> 2) * 64 + (c8 & 3) * 8 + 32, u[0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = activation<T, ACT>(g[0][j]) * u[0][j];      // (of the sums, not of what is kept of them)
                store_streamed<T>((T*)P.out + m * width + n, v);
                if (P.out2) {
                    store_streamed<T>((T*)P.out2 + m * 2 * width + n, g[0]);
                    store_streamed<T>((T*)P.out2 + m * 2 * width + width + n, u[0]);
                }
                continue;
            }
            take(row, 8 * c8, v);
            if constexpr (FORM == STORE) store_values<T, 8>((T*)P.out + m * width + n, v);
            if constexpr (FORM == PART) store_values<float, 8>((float*)P.out + ((long long)split * P.M + m) * width + n, v);
            if constexpr (FORM == DACT) {
                float h[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float c, d;
                    activation<T, ACT>(g[i][j], c, d);
                    h[j] = c * u[i][j];
                    g[i][j] = v[j] * u[i][j] * d;
                    u[i][j] = v[j] * c;
                }
                store_streamed<T>((T*)P.out + m * width + n, h);
                store_streamed<T>((T*)P.out2 + m * 2 * width + n, g[i]);
                store_streamed<T>((T*)P.out2 + m * 2 * width + width + n, u[i]);
            }
        }
    }
    }
}

template <typename T, int MB, int WM, int WN, int KB, int RING, bool QA, bool PA, Form FORM, int ACT>
__global__ void __launch_bounds__(64 * WM * WN, 2) ffn_gemm_kernel(const FfnParams P) {
    ffn_tile<T, MB, WM, WN, KB, RING, QA, PA, FORM, ACT>(P, blockIdx.x);
}
// Two products in one launch, the second one's workgroups from block `first` on (a multiple of 8)
struct FfnPair {
    FfnParams a, b;
    int first;
};
template <typename T, int MB, int WM, int WN, int KB, int RING>
__global__ void __launch_bounds__(64 * WM * WN, 2) ffn_outer_pair_kernel(const FfnPair P) {
    const bool second = (int)blockIdx.x >= P.first;
    const FfnParams& R = second ? P.b : P.a;
    const int block = blockIdx.x - (second ? P.first : 0);
    if (block >= (int)R.tiles.d * R.splits) return;      // (fills up to `first`)
    ffn_tile<T, MB, WM, WN, KB, RING, true, true, PART, 0>(R, block);
}

long long tiles_of(long long n, int tile) { return (n + tile - 1) / tile; }

// what the kernel needs to find its tile (the plan has seen to it that a launch holds them)
void number_tiles(FfnParams* P, int bm, int cols, int bn, int ks) {
    P->mt = (int)tiles_of(P->M, bm);
    P->nt = (int)tiles_of(cols, bn);
    const long long tiles = (long long)P->mt * P->nt, steps = tiles_of(P->K, ks);
    if (P->splits < 1) P->splits = 1;
    P->per = (int)(steps / P->splits);
    P->extra = (int)(steps % P->splits);
    P->tiles = make_div((uint32_t)tiles);
    P->band = make_div(4u * P->nt);
    P->last = make_div(P->mt % 4 ? P->mt % 4 : 4);
}
// Once for each device (bits of `done`), as the attribute belongs to the current one; a second thread racing here repeats an idempotent call
template <class Kernel>
int allow_lds(Kernel kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const uint64_t bit = 1ull << (dev & 63);
    if (e == hipSuccess && dev < 64 && done & bit) return MI3D_OK;
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) {
        note_hip_error(e);
        return MI3D_ERR_HIP;
    }
    if (dev < 64) done |= bit;
    return MI3D_OK;
}

template <typename T, int MB, int WM, int WN, int KB, int RING, bool QA, bool PA, Form FORM, int ACT>
int launch(FfnParams P, hipStream_t s) {
    constexpr int BM = 32 * MB * WM, BN = 64 * WN, LDS = RING * (BM + BN) * KB;
    number_tiles(&P, BM, FORM == GATE ? P.F : P.N, FORM == GATE ? BN / 2 : BN, KB / sizeof(T));
    const auto kernel = ffn_gemm_kernel<T, MB, WM, WN, KB, RING, QA, PA, FORM, ACT>;
    static std::atomic<uint64_t> allowed{0};
    const int st = allow_lds(kernel, LDS, allowed);
    if (st) return st;
    kernel<<<P.tiles.d * P.splits, 64 * WM * WN, LDS, s>>>(P);
    return check_launch();
}
template <typename T, int MB, int WM, int WN, int KB, int RING>
int launch_pair(FfnPair P, hipStream_t s) {
    constexpr int BM = 32 * MB * WM, BN = 64 * WN, LDS = RING * (BM + BN) * KB;
    number_tiles(&P.a, BM, P.a.N, BN, KB / sizeof(T));
    number_tiles(&P.b, BM, P.b.N, BN, KB / sizeof(T));
    P.first = (int)(P.a.tiles.d * P.a.splits + 7) / 8 * 8;
    const auto kernel = ffn_outer_pair_kernel<T, MB, WM, WN, KB, RING>;
    static std::atomic<uint64_t> allowed{0};
    const int st = allow_lds(kernel, LDS, allowed);
    if (st) return st;
    kernel<<<P.first + P.b.tiles.d * P.b.splits, 64 * WM * WN, LDS, s>>>(P);
    return check_launch();
}

// ---- which kernel, and into how many parts the contraction goes -----------------------------------------------------------
//
// The time of a product on tiles is rounds of workgroups (one or two on a compute unit), each of which takes a fixed time (first
// loads, results) and a time for every 128 bytes of k; less where it has its compute unit for itself.  Microseconds, measured over
// 300 to 27648 rows, 200 to 4096 channels and F 520 to 8192 (LARGE, MIDDLE, SMALL in us):
//   LARGE  256 x 256, 8 waves: fewest LDS reads a product, but alone on its unit: dx of 16384 x 1024 x 4096 240, 277, 373
//   MIDDLE 128 x 128: two on a unit, which cover some of each other's first loads and results, for short contractions:
//          first product of 27648 x 320 x 1280 87, 75, 102
//   SMALL  64 x 128: fills the chip with a quarter of the rows: second product of 3456 x 320 x 1280 33, 19, 11
//   FEW    no LDS (ffn_few.hip): small matrices and few rows: first product of 300 x 200 x 520 SMALL 6.3, FEW 4.4, of one row of
//          1024 x 4096 9.4 and 5.8
enum Tile { LARGE, MIDDLE, SMALL, FEW };
struct TileTimes {
    int bm, bn, threads, per_cu;
    double fixed, dact, alone, shared;      // per round, the same for the data gradient's first product; per 128 bytes of k
};
constexpr TileTimes TIMES_BF16[3] = {{256, 256, 512, 1, 12.0, 34.0, 1.6, 1.6}, {128, 128, 256, 2, 4.8, 14.0, 0.70, 1.09}, {64, 128, 256, 2, 3.7, 8.6, 0.38, 0.68}};
constexpr TileTimes TIMES_F32[3] = {{256, 256, 512, 1, 12.0, 34.0, 7.8, 7.8}, {128, 128, 256, 2, 4.8, 14.0, 2.2, 3.7}, {64, 128, 256, 2, 3.7, 8.6, 1.2, 2.1}};

struct Plan {
    Tile tile;
    int splits;
    double us;
    bool fits() const { return us < 1e30; }      // false: no tiles of which a launch holds as many as it takes
};
// (a launch counts its threads in 32 bits)
constexpr long long MOST_THREADS = (1ll << 31) - 1;
// Slices of the parts that ffn_add_parts_kernel's threads take side by side
int slices_of(int parts) {
    int S = 1;
    while (S < 8 && 2 * S <= parts) S *= 2;
    return S;
}
double tiles_us(const TileTimes& t, bool dact, long long tiles, double steps) {
    const long long cus = cu_count(), slots = t.per_cu * cus, rest = tiles % slots;
    const double fixed = dact ? t.dact : t.fixed;
    return (double)(tiles / slots) * (fixed + steps * t.shared) + (rest == 0 ? 0.0 : rest <= cus ? fixed + steps * t.alone : fixed + steps * t.shared);
}
// time of adding the parts of n sums, with the launch
double add_us(int splits, double n) { return splits > 1 ? 5.0 + (splits + 1.0) * 4.0 * n / 5e6 : 0.0; }
// cols: columns of D that tiles cover (GATE: of both halves).  most_parts 1: the contraction is not split.  M2 x cols2: a second product
// with the same contraction in the same launch
Plan plan(Form form, int e, long long M, long long cols, long long K, int most_parts, long long M2 = 0, long long cols2 = 0) {
    Plan best{MIDDLE, 1, 1e30};
    const double steps = (double)tiles_of(K * e, 128);
    for (int i = e == 2 ? 0 : 1; i < 3; ++i) {      // (fp32: LARGE has nothing to save, the matrix instructions take eight times longer)
        const TileTimes& t = (e == 2 ? TIMES_BF16 : TIMES_F32)[i];
        const long long tiles = tiles_of(M, t.bm) * tiles_of(cols, t.bn) + tiles_of(M2, t.bm) * tiles_of(cols2, t.bn);
        const long long n = M * cols + M2 * cols2;
        for (int s = 1; s <= most_parts && (s == 1 || s * 4 <= steps); s += s < 8 ? 1 : s / 4) {
            // (up to 7 workgroups between two products, one more in each addition)
            if ((tiles * s + 7) * t.threads > MOST_THREADS || (s > 1 && (n / 8 * slices_of(s) + 512) > MOST_THREADS)) continue;
            const double us = tiles_us(t, form == DACT, tiles * s, steps / s) + add_us(s, (double)n);
            if (us < best.us) best = Plan{(Tile)i, s, us};
        }
    }
    if (form == GATE || form == STORE) {
        const double us = few_rows_us(e == 2, M, K, form == GATE ? cols / 2 : cols);
        if (us < best.us) best = Plan{FEW, 1, us};
    }
    return best;
}
constexpr int MOST_PARTS = 64;

template <typename T, bool QA, bool PA, Form FORM, int ACT>
int on_tiles(const FfnParams& P, Tile tile, hipStream_t s) {
    if constexpr (sizeof(T) == 2)
        if (tile == LARGE) return launch<T, 4, 2, 4, 64, 4, QA, PA, FORM, ACT>(P, s);
    if (tile == MIDDLE) return launch<T, 2, 2, 2, 128, 2, QA, PA, FORM, ACT>(P, s);
    return launch<T, 1, 2, 2, 128, 3, QA, PA, FORM, ACT>(P, s);
}
template <typename T, bool QA, bool PA, Form FORM>
int gemm(const FfnParams& P, Tile tile, hipStream_t s, int act = MI3D_ACT_SILU) {
    if constexpr (FORM == GATE || FORM == DACT)
        if (act == MI3D_ACT_GELU) return on_tiles<T, QA, PA, FORM, MI3D_ACT_GELU>(P, tile, s);
    return on_tiles<T, QA, PA, FORM, MI3D_ACT_SILU>(P, tile, s);
}

// Sums of the parts of a contraction, rounded to the result's type; of two results one behind the other.  A workgroup has 256 / S groups
// of eight values: thread (slice, group) adds parts slice, slice + S, ..., and the S sums are added in order.
template <typename T>
struct Parts {
    const float* part;      // [parts][n]
    T* out;
    long long n;
    int blocks;
};
template <typename T>
__global__ void __launch_bounds__(256) ffn_add_parts_kernel(const Parts<T> a, const Parts<T> b, int parts, int S) {
    __shared__ float red[256 * 8];
    const bool second = (int)blockIdx.x >= a.blocks;
    const Parts<T>& R = second ? b : a;
    const int t = threadIdx.x, groups = 256 / S, slice = t / groups, g = t % groups;
    const long long at = ((long long)blockIdx.x - (second ? a.blocks : 0)) * groups * 8;
    float v[8] = {}, o[8];
    if (at + 8 * g < R.n)
        for (int p = slice; p < parts; p += S) {
            load_values<float, 8>(R.part + p * R.n + at + 8 * g, o);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += o[j];
        }
    if (S == 1) {
        if (at + 8 * g < R.n) store_values<T, 8>(R.out + at + 8 * g, v);
        return;
    }
    store_values<float, 8>(red + t * 8, v);
    __syncthreads();
    for (int i = t; i < groups * 8; i += 256) {
        if (at + i >= R.n) break;
        o[0] = red[i];
        for (int p = 1; p < S; ++p) o[0] += red[p * groups * 8 + i];
        const float r[1] = {o[0]};
        store_values<T, 1>(R.out + at + i, r);
    }
}
template <typename T>
int add_parts(const float* part, T* out, long long n, const float* part2, T* out2, long long n2, int parts, hipStream_t s) {
    const int S = slices_of(parts);
    const int values = 256 / S * 8;
    const Parts<T> a = {part, out, n, (int)tiles_of(n, values)}, b = {part2, out2, n2, (int)tiles_of(n2, values)};
    ffn_add_parts_kernel<T><<<(unsigned)(a.blocks + b.blocks), 256, 0, s>>>(a, b, parts, S);
    return check_launch();
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
// The plans of a pass.  pair: both weight gradients in one launch, else one after the other with parts of their own (additions of the parts
// included, 16384 x 1024 x 4096: 432 us together, 404 apart; 27000 x 256 x 1024: 62 and 74)
struct Plans {
    Plan first, second;
    bool pair;
    bool fit() const { return first.fits() && second.fits(); }
};
Plans make_plans(const Desc& d, int pass) {
    if (pass == MI3D_PASS_FWD) return Plans{plan(GATE, d.e, d.rows, 2 * d.F, d.C, 1), plan(STORE, d.e, d.rows, d.O, d.F, MOST_PARTS), false};
    if (pass == MI3D_PASS_DGRAD) return Plans{plan(DACT, d.e, d.rows, d.F, d.O, 1), plan(PART, d.e, d.rows, d.C, 2 * d.F, MOST_PARTS), false};
    const Plan both = plan(PART, d.e, 2 * d.F, d.C, d.rows, MOST_PARTS, d.O, d.F);
    const Plan first = plan(PART, d.e, 2 * d.F, d.C, d.rows, MOST_PARTS), second = plan(PART, d.e, d.O, d.F, d.rows, MOST_PARTS);
    if (both.us <= first.us + second.us + 3.0) return Plans{both, both, true};
    return Plans{first, second, false};
}
// A call asks twice (its workspace, its kernels) and the weighing takes 1 to 3 us, a quarter of what one row takes in all: a thread keeps
// the last ones, by everything that they depend on.
Plans plans_of(const Desc& d, int pass) {
    struct Slot {
        long long rows;
        int C, F, O, e, pass, cus;
        Plans plans;
    };
    static thread_local Slot slots[16];      // (C = 0: none)
    const int cus = cu_count();
    uint64_t h = (uint64_t)d.rows * 3 + pass;
    for (int v : {d.C, d.F, d.O, d.e}) h = h * 0x9E3779B97F4A7C15ull + (uint32_t)v;
    Slot& s = slots[h * 0x9E3779B97F4A7C15ull >> 60];
    if (s.rows != d.rows || s.C != d.C || s.F != d.F || s.O != d.O || s.e != d.e || s.pass != pass || s.cus != cus)
        s = Slot{d.rows, d.C, d.F, d.O, d.e, pass, cus, make_plans(d, pass)};
    return s.plans;
}
size_t parts_bytes(int splits, long long M, long long N) { return splits > 1 ? (size_t)splits * M * N * 4 : 0; }
bool usable(const void* p) { return p && aligned16(p); }

size_t workspace(const Desc& d, int pass) {
    if (pass < MI3D_PASS_FWD || pass > MI3D_PASS_WGRAD || (!d.rows && pass != MI3D_PASS_WGRAD)) return 0;
    const Plans p = plans_of(d, pass);
    if (!p.fit()) return 0;
    if (pass == MI3D_PASS_FWD) return round256((size_t)d.rows * d.F * d.e) + parts_bytes(p.second.splits, d.rows, d.O);      // h, parts of y
    if (pass == MI3D_PASS_DGRAD) return parts_bytes(p.second.splits, d.rows, d.C);
    const size_t n1 = parts_bytes(p.first.splits, 2 * d.F, d.C), n2 = parts_bytes(p.second.splits, d.O, d.F);
    return p.pair ? n1 + n2 : n1 > n2 ? n1 : n2;
}

template <typename T>
int gate(const Desc& d, const void* x, const void* w1, void* h, void* gu, hipStream_t s) {
    const Plan p = plans_of(d, MI3D_PASS_FWD).first;
    if (p.tile == FEW) return few_rows_product(sizeof(T) == 2, true, x, w1, d.rows, d.C, d.F, d.act, h, gu, s);
    FfnParams P{};
    P.q = x; P.p = w1; P.M = d.rows; P.K = d.C; P.N = d.F; P.qp = d.C; P.pp = d.C; P.F = d.F;
    P.out = h; P.out2 = gu;
    return gemm<T, false, false, GATE>(P, p.tile, s, d.act);
}
// D of P's operands, by way of its parts where the plan has some
template <typename T, bool PA>
int rows_product(FfnParams P, const Plan& p, void* out, void* parts, hipStream_t s) {
    P.splits = p.splits;
    P.out = p.splits > 1 ? parts : out;
    if (p.splits == 1) return gemm<T, false, PA, STORE>(P, p.tile, s);
    const int st = gemm<T, false, PA, PART>(P, p.tile, s);
    return st ? st : add_parts<T>((const float*)parts, (T*)out, P.M * P.N, nullptr, nullptr, 0, p.splits, s);
}
template <typename T>
int project(const Desc& d, void* ws, const void* w2, void* y, hipStream_t s) {
    const Plan p = plans_of(d, MI3D_PASS_FWD).second;
    if (p.tile == FEW) return few_rows_product(sizeof(T) == 2, false, ws, w2, d.rows, d.F, d.O, 0, y, nullptr, s);
    FfnParams P{};
    P.q = ws; P.p = w2; P.M = d.rows; P.K = d.F; P.N = d.O; P.qp = d.F; P.pp = d.F;
    return rows_product<T, false>(P, p, y, (char*)ws + round256((size_t)d.rows * d.F * d.e), s);
}
template <typename T>
int dgrad(const Desc& d, const void* dy, const void* w1, const void* w2, const void* gu, void* dgu, void* h, void* dx, void* ws, hipStream_t s) {
    FfnParams P{};
    P.q = dy; P.p = w2; P.M = d.rows; P.K = d.O; P.N = d.F; P.qp = d.O; P.pp = d.F;
    P.out = h; P.out2 = dgu; P.gu = gu;
    const Plans p = plans_of(d, MI3D_PASS_DGRAD);
    const int st = gemm<T, false, true, DACT>(P, p.first.tile, s, d.act);
    if (st) return st;
    FfnParams R{};
    R.q = dgu; R.p = w1; R.M = d.rows; R.K = 2 * d.F; R.N = d.C; R.qp = 2 * d.F; R.pp = d.C;
    return rows_product<T, true>(R, p.second, dx, ws, s);
}
template <typename T>
int wgrad(const Desc& d, const void* x, const void* dgu, const void* h, const void* dy, float* dw1, float* dw2, void* ws, hipStream_t s) {
    const Plans p = plans_of(d, MI3D_PASS_WGRAD);
    const long long n1 = 2ll * d.F * d.C, n2 = (long long)d.O * d.F;
    float* parts = (float*)ws;
    FfnPair P{};
    P.a.q = dgu; P.a.p = x; P.a.M = 2 * d.F; P.a.K = d.rows; P.a.N = d.C; P.a.qp = 2 * d.F; P.a.pp = d.C; P.a.splits = p.first.splits;
    P.b.q = dy; P.b.p = h; P.b.M = d.O; P.b.K = d.rows; P.b.N = d.F; P.b.qp = d.O; P.b.pp = d.F; P.b.splits = p.second.splits;
    P.a.out = p.first.splits > 1 ? parts : dw1;
    P.b.out = p.second.splits > 1 ? parts + (p.pair ? p.first.splits * n1 : 0) : dw2;
    int st;
    if (!p.pair) {
        st = gemm<T, true, true, PART>(P.a, p.first.tile, s);
        if (!st && p.first.splits > 1) st = add_parts<float>(parts, dw1, n1, nullptr, nullptr, 0, p.first.splits, s);
        if (!st) st = gemm<T, true, true, PART>(P.b, p.second.tile, s);
        return st || p.second.splits == 1 ? st : add_parts<float>(parts, dw2, n2, nullptr, nullptr, 0, p.second.splits, s);
    }
    if (sizeof(T) == 2 && p.first.tile == LARGE) st = launch_pair<uint16_t, 4, 2, 4, 64, 4>(P, s);
    else if (p.first.tile == MIDDLE) st = launch_pair<T, 2, 2, 2, 128, 2>(P, s);
    else st = launch_pair<T, 1, 2, 2, 128, 3>(P, s);
    return st || p.first.splits == 1 ? st : add_parts<float>(parts, dw1, n1, parts + p.first.splits * n1, dw2, n2, p.first.splits, s);
}

}  // namespace
}  // namespace mi3d

using namespace mi3d;

extern "C" {

size_t mi3d_ffn_workspace_bytes(const mi3d_ffn_desc* desc, int pass) {
    Desc d;
    return make(desc, &d) == MI3D_OK ? workspace(d, pass) : 0;
}

int mi3d_ffn_kernel_detail(const mi3d_ffn_desc* desc, int pass, char* buf, size_t buf_len) {
    Desc d;
    const int st = make(desc, &d);
    if (st) return st;
    if (!buf || !buf_len || pass < MI3D_PASS_FWD || pass > MI3D_PASS_WGRAD) return MI3D_ERR_INVALID_ARG;
    static const char* const names[4] = {"tiles_256x256", "tiles_128x128", "tiles_64x128", "few_rows"};
    const Plans p = plans_of(d, pass);
    if (!p.fit()) return MI3D_ERR_UNSUPPORTED;
    const char *first = names[p.first.tile], *second = names[p.second.tile];
    if (pass != MI3D_PASS_WGRAD) snprintf(buf, buf_len, "%s, %s parts %d", first, second, p.second.splits);
    else if (p.pair) snprintf(buf, buf_len, "pair %s parts %d", first, p.first.splits);
    else snprintf(buf, buf_len, "%s parts %d, %s parts %d", first, p.first.splits, second, p.second.splits);
    return MI3D_OK;
}

int mi3d_ffn_gate(const mi3d_ffn_desc* desc, const void* x, const void* w1, void* h, void* gu, void* stream) {
    Desc d;
    const int st = make(desc, &d);
    if (st) return st;
    if (!usable(w1) || !aligned16(x) || !aligned16(h) || !aligned16(gu)) return MI3D_ERR_INVALID_ARG;
    if (d.rows == 0) return MI3D_OK;
    if (!x || !h) return MI3D_ERR_INVALID_ARG;
    if (!plans_of(d, MI3D_PASS_FWD).first.fits()) return MI3D_ERR_UNSUPPORTED;
    return d.e == 2 ? gate<uint16_t>(d, x, w1, h, gu, (hipStream_t)stream) : gate<float>(d, x, w1, h, gu, (hipStream_t)stream);
}

int mi3d_ffn_fwd(const mi3d_ffn_desc* desc, const void* x, const void* w1, const void* w2, void* y, void* gu, void* ws, size_t ws_bytes, void* stream) {
    Desc d;
    int st = make(desc, &d);
    if (st) return st;
    if (!usable(w1) || !usable(w2) || !aligned16(x) || !aligned16(y) || !aligned16(gu) || !aligned16(ws)) return MI3D_ERR_INVALID_ARG;
    if (d.rows == 0) return MI3D_OK;
    if (!x || !y) return MI3D_ERR_INVALID_ARG;
    if (!plans_of(d, MI3D_PASS_FWD).fit()) return MI3D_ERR_UNSUPPORTED;
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
    if (!plans_of(d, MI3D_PASS_DGRAD).fit()) return MI3D_ERR_UNSUPPORTED;
    const size_t need = workspace(d, MI3D_PASS_DGRAD);
    if (need && (!ws || ws_bytes < need)) return MI3D_ERR_WORKSPACE;
    return d.e == 2 ? dgrad<uint16_t>(d, dy, w1, w2, gu, dgu, h, dx, ws, (hipStream_t)stream) : dgrad<float>(d, dy, w1, w2, gu, dgu, h, dx, ws, (hipStream_t)stream);
}

int mi3d_ffn_wgrad(const mi3d_ffn_desc* desc, const void* x, const void* dgu, const void* h, const void* dy, float* dw1, float* dw2,
                   void* ws, size_t ws_bytes, void* stream) {
    Desc d;
    const int st = make(desc, &d);
    if (st) return st;
    if (!usable(dw1) || !usable(dw2) || !aligned16(x) || !aligned16(dgu) || !aligned16(h) || !aligned16(dy) || !aligned16(ws)) return MI3D_ERR_INVALID_ARG;
    if (d.rows && (!x || !dgu || !h || !dy)) return MI3D_ERR_INVALID_ARG;
    if (!plans_of(d, MI3D_PASS_WGRAD).fit()) return MI3D_ERR_UNSUPPORTED;
    const size_t need = workspace(d, MI3D_PASS_WGRAD);
    if (need && (!ws || ws_bytes < need)) return MI3D_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    return d.e == 2 ? wgrad<uint16_t>(d, x, dgu, h, dy, dw1, dw2, ws, s) : wgrad<float>(d, x, dgu, h, dy, dw1, dw2, ws, s);
}

}  // extern "C"
