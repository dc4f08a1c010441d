// The split kernel of kv_attention.cuh for one element type.
#pragma once

#include "async_copy.cuh"
#include "kv_attention.cuh"

namespace mosaic {
namespace {

// Set when a bounded wait ran out (read by attend_status).
__device__ unsigned int g_attend_error;

// 16 bytes, or zeros where !ok (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Arrives (for this lane, one of the barrier's count) when the lane's copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float lds(uint32_t a) {
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(a) : "memory");
    return x;
}
// d += a b (mma0: d = a b), 16 x 8 x 16 (16-bit types) or 16 x 8 x 8 (tf32).
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma0(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma0(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma0(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
// x, y rounded to the type and packed (x lower); and back.
__device__ __forceinline__ uint32_t pack2(float x, float y, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float x, float y, __half) {
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack2(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t v, __half) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}
// fp16: a term is kept times 2^12 of the next greater one's scale, which keeps
// it clear of subnormals: of an x of up to 2^15 a term's rest is 8 at most.
template <class T> constexpr float kStep = 1.0f;
template <> constexpr float kStep<__half> = 4096.0f;
// x, y -> terms t[0] (the least) .. t[N-1] (the greatest), packed.
template <class T, int N>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        t[i] = pack2(x, y, T());
        if (i) {
            const float2 v = unpack2(t[i], T());
            x = (x - v.x) * kStep<T>, y = (y - v.y) * kStep<T>;
        }
    }
}
// fp32 as two tf32 terms, the upper one rounded to nearest (the lower one then
// has either sign, and what is left out averages out); the lower one's own tail
// (2^-23) is cut by the tensor core.
__device__ __forceinline__ uint32_t tf32_high(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }
__device__ __forceinline__ uint32_t tf32_low(float x, uint32_t high) {
    return __float_as_uint(x - __uint_as_float(high));
}

template <class T> constexpr int kTerms = sizeof(T) == 4 ? 2 : 3;
template <> constexpr int kTerms<__half> = 2;
// Probabilities, and with them sums and outputs of a job, are kept times this:
// two fp16 terms then hold 22 bits of one down to 2^-29.
template <class T> constexpr float kScaleP = 1.0f;
template <> constexpr float kScaleP<__half> = 0x1p15f;
// Those below (scaled: the least normal fp16) take a pass of their own, 2^29
// times as large, and those below 2^-58 a third.
constexpr float kLeastP = 0x1p-14f, kPassP = 0x1p29f;

constexpr int kTogether = 4;   // chains of products at a time
constexpr int kLookup = 4 * 128 + 32;   // bytes of a producer's page ids and live slots

// DP: head_dim padded to 64, 128 or 256.  NT: tiles of 8 query heads.
template <class T, int DP, int NT>
struct Shape {
    static constexpr int kES = sizeof(T), kRow = DP * kES, kChunks = kRow / 16;
    // A stage holds a unit: K and V of kUnit rows, 16 a consumer warp (slots of
    // a.hpu heads).  8 consumer warps an SM, as two blocks or (with twice the outputs and queries) one;
    // fewer where rows are long.
    static constexpr int kWarps = kRow == 1024 ? 2 : NT == 2 && kRow <= 256 ? 8 : 4;
    static constexpr int kUnit = 16 * kWarps, kStage = 2 * kUnit * kRow;
    static constexpr int kStages = kRow == 128 ? 4 : (NT == 2 && DP == 256) ? 2 : 3;
    static constexpr int kSlots = kWarps == 2 || (NT == 2 && kRow >= 512) ? 1 : 2;   // warps' results at a time
    static constexpr int kK = kES == 4 ? 8 : 16, kSteps = DP / kK;    // channels of a product step
    static constexpr int kHeads = 8 * NT, kPitch = DP + 4;
    static constexpr int kQWords = kSteps * NT * kTerms<T> * 2 * 32;  // query fragments
    // Queries stay in registers where they fit beside the outputs.
    static constexpr int kQRegs = kSteps * NT * kTerms<T> * 2;
    static constexpr bool kQReg = kQRegs <= 48 || (kQRegs <= 64 && NT == 1 && kRow == 512);
    static constexpr int kQHeads = kQReg ? 0 : 1;   // else in shared memory, of one head
    // Shared memory: the ring, the results of some warps, page ids and live
    // slots of the producers' groups, the queries' fragments, barriers and so on.
    static constexpr int kRing = kStages * kStage;
    static constexpr int kMerge = 4 * kSlots * kHeads * (kPitch + 2);
    static constexpr int kIds = 2 * kLookup;
    static constexpr int kQAt = kRing + kMerge + kIds, kMiscAt = kQAt + 4 * kQWords * kQHeads;
    static constexpr int kMisc = 512 + 8 * kHeads * (kQReg ? kWarps : kQHeads);
    static constexpr int kBytes = kMiscAt + kMisc;
    static constexpr int kFit = 228 * 1024 / (kBytes + 1024), kBlocks = kFit < 3 ? kFit : 3;   // blocks an SM
    static_assert(kBytes <= 227 * 1024, "shared memory");
};
constexpr int kProducers = 2;   // warps that copy

// A stage: K, then V of a unit; each in blocks of 128 bytes of all its rows,
// 16-byte chunk c of row r at chunk c ^ (r % 8) of its block (the tensor copies'
// 128-byte swizzle).  8 rows of a chunk are conflict-free (ldmatrix), and so are
// 8 words of rows r, r + 2, r + 4 and r + 6.
template <int BLOCK>   // bytes of a block of all rows
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    return (uint32_t)((c >> 3) * BLOCK + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

template <class T, int DP, int NT>
struct Warp {
    using S = Shape<T, DP, NT>;
    static constexpr int kTermsN = kTerms<T>, kBlock = 128 * S::kUnit;
    float m[NT][2], l[NT][2], o[NT][DP / 16][4];   // of heads 2t, 2t + 1 of each tile
    uint32_t qr[S::kQReg ? S::kSteps * NT * kTermsN * 2 : 1];
    float unscale[NT][2];                          // fp16: what undoes the queries' scaling

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = minus_inf(), l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][i][j] = 0.0f;
        }
    }

    // Fragments of the job's queries: column (head) lane / 4, rows (channels)
    // by the step.  `rows`: query heads of the job; the rest count as zeros.
    __device__ __forceinline__ void queries(const float *q, int D, int rows, float scale2, uint32_t *qs) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool in = 8 * n + g < rows;
            const float *x = q + (int64_t)(8 * n + g) * D;
            float v[S::kSteps][S::kES == 4 ? 2 : 4];   // all loads before their use
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k)
#pragma unroll
                for (int j = 0; j < (S::kES == 4 ? 2 : 4); ++j) {
                    const int d = S::kES == 4 ? 8 * k + 4 * j + t : 16 * k + 8 * (j >> 1) + 2 * t + (j & 1);
                    v[k][j] = in && d < D ? x[d] * scale2 : 0.0f;
                }
            if constexpr (sizeof(T) == 2 && kTermsN == 2) {
                float top = 0.0f;
#pragma unroll
                for (int k = 0; k < S::kSteps; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(v[k][j]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // Largest |q| to [2^14, 2^15); nothing to scale in zeros, NaN and infinities.
                int e = (int)(__float_as_uint(top) >> 23) - 127;
                e = e == 128 || top == 0.0f ? 14 : e < -100 ? -100 : e;
                const float up = __uint_as_float((uint32_t)(14 - e + 127) << 23);
                const float down = __uint_as_float((uint32_t)(e - 14 + 127) << 23);
                unscale[n][0] = __shfl_sync(0xffffffffu, down, 8 * t);
                unscale[n][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
#pragma unroll
                for (int k = 0; k < S::kSteps; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[k][j] *= up;
            }
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k) {
                uint32_t f[kTermsN][2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    if constexpr (sizeof(T) == 4) {
                        f[1][b] = tf32_high(v[k][b]);
                        f[0][b] = tf32_low(v[k][b], f[1][b]);
                    } else {
                        uint32_t s[kTermsN];
                        split2<T, kTermsN>(v[k][2 * b], v[k][2 * b + 1], s);
#pragma unroll
                        for (int i = 0; i < kTermsN; ++i) f[i][b] = s[i];
                    }
                }
#pragma unroll
                for (int i = 0; i < kTermsN; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int at = ((k * NT + n) * kTermsN + i) * 2 + b;
                        if constexpr (S::kQReg) qr[at] = f[i][b];
                        else qs[at * 32 + lane] = f[i][b];
                    }
            }
        }
    }
    __device__ __forceinline__ uint32_t query(const uint32_t *qs, int k, int n, int i, int b) const {
        const int at = ((k * NT + n) * kTermsN + i) * 2 + b;
        if constexpr (S::kQReg) return qr[at];
        else return qs[at * 32 + (threadIdx.x & 31)];
    }

    // Sums of products of one term, on the scale of the next greater one.
    template <int N>
    static __device__ __forceinline__ void next_term(float (&c)[N][NT][4]) {
        if constexpr (kStep<T> != 1.0f) {
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[k][n][j] *= 1.0f / kStep<T>;
        }
    }

    // One tile of 16 slots, K rows at `tile` and V rows at `vbase`; bit r of
    // `live`: slot r counts.  `sc`: where the scores of slot 0 and the job's
    // first head go (a row of `pitch` words a head, `heads` of them), or null.
    __device__ __forceinline__ void tile(uint32_t tile, uint32_t vbase, uint32_t live, const uint32_t *qs, float *sc, int64_t pitch,
                                         int heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float s[NT][4];
        const uint32_t base = tile + chunk_at<kBlock>(lane & 15, lane >> 4);
        // kTogether independent chains at a time (one alone waits out the latency
        // of each of its products), each over two steps, the least terms first.
        constexpr int KT = kTogether / NT, KB = 2 * KT < S::kSteps ? 2 * KT : S::kSteps;
        static_assert(S::kSteps % KB == 0 && KB % KT == 0, "steps");
#pragma unroll
        for (int k0 = 0; k0 < S::kSteps; k0 += KB) {
            uint32_t a[KB][4];
            float c[KT][NT][4];
#pragma unroll
            for (int k = 0; k < KB; ++k) ldm4(a[k], (base ^ (2 * (k0 + k) % 8 << 4)) + (2 * (k0 + k) / 8) * kBlock);
            auto product = [&](bool first, int k, const uint32_t (&x)[4], int i) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t b0 = query(qs, k0 + k, n, i, 0), b1 = query(qs, k0 + k, n, i, 1);
                    if (first) mma0(c[k % KT][n], x, b0, b1, T());
                    else mma(c[k % KT][n], x, b0, b1, T());
                }
            };
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    uint32_t lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = __uint_as_float(a[k][i]);
                        a[k][i] = tf32_high(v);
                        lo[i] = tf32_low(v, a[k][i]);
                    }
                    product(k < KT, k, lo, 1);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < KB; ++k) product(false, k, a[k], i);
            } else {
#pragma unroll
                for (int i = 0; i < kTermsN; ++i) {
#pragma unroll
                    for (int k = 0; k < KB; ++k) product(i == 0 && k < KT, k, a[k], i);
                    if (i + 1 < kTermsN) next_term(c);
                }
            }
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][j] = k0 + k == 0 ? c[k][n][j] : s[n][j] + c[k][n][j];
        }
        const bool up = live >> g & 1, dn = live >> (g + 8) & 1;
        float alpha[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2 && kTermsN == 2) s[n][j] *= unscale[n][j & 1];
                // An infinite key: the terms of a query sum to either infinity or NaN, by their signs.
                s[n][j] = (j < 2 ? up : dn) ? finite_or_nan(s[n][j]) : minus_inf();
            }
            if (sc) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int h = 8 * n + 2 * t + (j & 1);   // 8 slots of 4 heads a store: whole sectors
                    if (h < heads) sc[h * pitch + g + (j & 2) * 4] = s[n][j];
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = fmaxf(s[n][j], s[n][2 + j]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                top = fmaxf(top, m[n][j]);
                alpha[n][j] = power2(m[n][j] - top);
                m[n][j] = top;
                s[n][j] = power2(s[n][j] - top) * kScaleP<T>;
                s[n][2 + j] = power2(s[n][2 + j] - top) * kScaleP<T>;
                l[n][j] = fmaf(l[n][j], alpha[n][j], s[n][j] + s[n][2 + j]);
            }
        }
        if constexpr (sizeof(T) == 2) {
            // Slots (lane / 16) * 8 + lane % 8, channels 16 i + 8 (lane / 8 % 2).
            const uint32_t at = vbase + chunk_at<kBlock>((lane >> 4) * 8 + (lane & 7), lane >> 3 & 1);
            int pass = 0;
            float up = 1.0f;   // fp16: of the pass
            if constexpr (kScaleP<T> != 1.0f) {
                auto below = [&](float least) {   // any of (0, least)?
                    bool any = false;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) any |= __float_as_uint(s[n][j]) - 1 < __float_as_uint(least) - 1;
                    return __any_sync(0xffffffffu, any);
                };
                if (below(kLeastP)) {   // the smallest first: outputs are scaled for them and back
                    pass = below(kLeastP / kPassP) ? 2 : 1;
                    up = pass == 2 ? kPassP * kPassP : kPassP;
#pragma unroll
                    for (int n = 0; n < NT; ++n) alpha[n][0] *= up, alpha[n][1] *= up;
                }
            }
            const int first = pass;
            do {
                uint32_t p16[NT][kTermsN][2];   // terms of P^T, as the product wants them
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float v[4] = {s[n][0], s[n][1], s[n][2], s[n][3]};
                    if (kScaleP<T> != 1.0f && first > 0) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            v[j] *= up;
                            if ((pass > 0 && v[j] >= kLeastP * kPassP) || (pass < first && v[j] < kLeastP)) v[j] = 0.0f;
                        }
                    }
                    uint32_t x[kTermsN], y[kTermsN];
                    split2<T, kTermsN>(v[0], v[1], x);
                    split2<T, kTermsN>(v[2], v[3], y);
#pragma unroll
                    for (int i = 0; i < kTermsN; ++i) p16[n][i][0] = transpose8(x[i]), p16[n][i][1] = transpose8(y[i]);
                }
#pragma unroll
                for (int i0 = 0; i0 < DP / 16; i0 += KT) {
                    uint32_t a[KT][4];
                    float c[KT][NT][4];
#pragma unroll
                    for (int i = 0; i < KT; ++i) {
                        ldm4t(a[i], (at ^ (2 * (i0 + i) % 8 << 4)) + (2 * (i0 + i) / 8) * kBlock);
                    }
#pragma unroll
                    for (int x = 0; x < kTermsN; ++x) {
#pragma unroll
                        for (int i = 0; i < KT; ++i)
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if (x == 0) mma0(c[i][n], a[i], p16[n][x][0], p16[n][x][1], T());
                                else mma(c[i][n], a[i], p16[n][x][0], p16[n][x][1], T());
                            }
                        if (x + 1 < kTermsN) next_term(c);
                    }
#pragma unroll
                    for (int i = 0; i < KT; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                o[n][i0 + i][j] = fmaf(o[n][i0 + i][j], alpha[n][j & 1], c[i][n][j]);
                }
                if constexpr (kScaleP<T> == 1.0f) break;
                up *= 1.0f / kPassP;
#pragma unroll
                for (int n = 0; n < NT; ++n) alpha[n][0] = alpha[n][1] = 1.0f / kPassP;
            } while (--pass >= 0);
        } else {
            // By step of 8 slots; the step's row t is slot 2t, row t + 4 slot 2t + 1.
            uint32_t ph[NT][2][2], pl[NT][2][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int from = (2 * t + b) * 4 + (g >> 1);
                        const float x = __shfl_sync(0xffffffffu, s[n][2 * k], from);
                        const float y = __shfl_sync(0xffffffffu, s[n][2 * k + 1], from);
                        const float v = g & 1 ? y : x;
                        ph[n][k][b] = tf32_high(v);
                        pl[n][k][b] = tf32_low(v, ph[n][k][b]);
                    }
            constexpr int IT = kTogether / NT / 2;   // two chains (steps) each
#pragma unroll
            for (int i0 = 0; i0 < DP / 16; i0 += IT) {
                float c[IT][NT][2][4];
                uint32_t hi[IT][2][4], lo[IT][2][4];
#pragma unroll
                for (int i = 0; i < IT; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int r = 8 * k + 2 * t + (j >> 1), ch = 4 * (i0 + i) + (g >> 2) + 2 * (j & 1);
                            hi[i][k][j] = __float_as_uint(lds(vbase + chunk_at<kBlock>(r, ch) + (g & 3) * 4));
                        }
#pragma unroll
                for (int i = 0; i < IT; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float v = __uint_as_float(hi[i][k][j]);
                            hi[i][k][j] = tf32_high(v);
                            lo[i][k][j] = tf32_low(v, hi[i][k][j]);
                        }
#pragma unroll
                for (int x = 0; x < 3; ++x)
#pragma unroll
                    for (int i = 0; i < IT; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                if (x == 0) mma0(c[i][n][k], lo[i][k], ph[n][k][0], ph[n][k][1], T());
                                else if (x == 1) mma(c[i][n][k], hi[i][k], pl[n][k][0], pl[n][k][1], T());
                                else mma(c[i][n][k], hi[i][k], ph[n][k][0], ph[n][k][1], T());
                            }
#pragma unroll
                for (int i = 0; i < IT; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            o[n][i0 + i][j] = fmaf(o[n][i0 + i][j], alpha[n][j & 1], c[i][n][0][j] + c[i][n][1][j]);
            }
        }
    }
};

// Work is counted in units; a job counts a.job_cost units more than it has, for
// what its queries, its merge and its output take.
//
// The jobs of a block, one after the other: a stretch of `left` counted units,
// from counted unit `at` of sequence i on.
struct Jobs {
    int64_t i, at, left;
    int r, b0, b1, nb, len;   // the job: number in its sequence, its units here, all its units, the sequence's length
    __device__ __forceinline__ bool next(const KvView &kv, const AttendArgs &a, int unit, int per_seq) {
        while (left > 0) {
            len = kv.length(a.lens, i, a.max_len);
            nb = (len + unit - 1) / unit;
            if (a.whole) {
                r = (int)at, b0 = 0, b1 = nb, left = 0;
                return true;
            }
            const int counted = nb + a.job_cost;
            if (nb == 0 || at >= (int64_t)counted * per_seq) {
                ++i, at = 0;
                continue;
            }
            r = (int)((uint32_t)at / (uint32_t)counted);   // a sequence counts below 2^31 units
            const int x0 = (int)at - r * counted, x1 = counted - x0 < left ? counted : x0 + (int)left;
            left -= x1 - x0, at += x1 - x0;
            b0 = max(0, x0 - a.job_cost), b1 = max(0, x1 - a.job_cost);
            if (b0 < b1) return true;
        }
        return false;
    }
    __device__ __forceinline__ int first(int unit) const { return b0 * unit; }
    __device__ __forceinline__ int last(int unit) const { return min(len, b1 * unit); }
};

// Counted units of the whole call (`total`), the stretch of part `part` of
// `parts`, and the sequence and offset of its beginning.  Every thread calls
// it; `sh` holds a word a warp and two more.
template <int THREADS>
__device__ __forceinline__ void find_place(const KvView &kv, const AttendArgs &a, int unit, int64_t per_seq, int part,
                                           int parts, int64_t &total, int64_t &u1, Jobs &jobs, long long *sh) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t seqs = kv.c.seqs;
    auto units = [&](int64_t i) -> long long {
        const int nb = i < seqs ? (kv.length(a.lens, i, a.max_len) + unit - 1) / unit : 0;
        return nb ? (long long)(nb + a.job_cost) * per_seq : 0;
    };
    long long mine = 0;
    for (int64_t i = tid; i < seqs; i += THREADS) mine += units(i);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, x);
    if (lane == 0) sh[w] = mine;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) total += sh[k];
    const long long u0 = total * part / parts;
    u1 = total * (part + 1) / parts;
    jobs.i = jobs.at = 0, jobs.left = u1 - u0;
    __syncthreads();
    if (u0 >= u1) return;
    long long before = 0;
    for (int64_t i0 = 0; i0 < seqs; i0 += THREADS) {
        const long long v = units(i0 + tid);
        long long x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sh[w] = x;
        __syncthreads();
        long long all = 0, pre = before;
#pragma unroll
        for (int k = 0; k < THREADS / 32; ++k) {
            if (k < w) pre += sh[k];
            all += sh[k];
        }
        const long long end = pre + x;
        if (u0 < end && u0 >= end - v) sh[THREADS / 32] = i0 + tid, sh[THREADS / 32 + 1] = u0 - (end - v);
        __syncthreads();
        before += all;
        if (u0 < before) break;
    }
    jobs.i = sh[THREADS / 32], jobs.at = sh[THREADS / 32 + 1];
    __syncthreads();
}

// What producers and consumers share beside the ring.
template <class T, int DP, int NT>
struct Pipe {
    using S = Shape<T, DP, NT>;
    uint64_t full[S::kStages], empty[S::kStages];
    uint16_t live[S::kStages][8];   // slots of the stage's tiles that count
    int unit[S::kStages];           // the stage's unit in its job; + kLastUnit: the job's last one here
    long long place[12];
    int aborted;
    float2 stats[S::kHeads * (S::kQReg ? S::kWarps : S::kQHeads)];   // whole jobs: for the weights
};
constexpr int kLastUnit = 1 << 30;

// A producer warp: copies unit by unit, through all jobs of the block.  Pages
// are looked up a group of units at a time, two groups (with a lower bound: and
// the positions, one group) before they are copied.
// TMA: tensor copies of rows that share a page, a lane's to issue; the first
// warp copies K and the second V of every unit, and units without a live slot
// are left out (but for a job's last, which ends it).  A lane looks up 8 slots
// at once.
// Else every lane copies 16 bytes at a time; the warps take turns at units and
// look up their own, a lane four single slots.
template <class T, int DP, int NT, bool TMA>
struct Producer {
    using S = Shape<T, DP, NT>;
    static constexpr int kSpan = TMA ? 256 : 128, kEach = TMA ? 1 : 4;   // rows of a group, look-ups of a lane
    static constexpr int kUnits = kSpan / S::kUnit, kHalves = S::kUnit / 16, kTurn = TMA ? 1 : kProducers;
    struct Group {
        int h, hb, s, end, units, low;   // first head, first slot, end of the job's slots, units, position bound
        int unit, of, base;              // number of its first unit in the job, of how many, units of all jobs before
        int64_t i;
    };
    const KvView &kv;
    const AttendArgs &a;
    const CUtensorMap *map;
    Pipe<T, DP, NT> &pipe;
    char *smem;
    const int per_seq, pw, lane, us, per_tile;   // us: slots of a unit; per_tile: 2^8 over the tiles of a head, rounded up
    int32_t *ids;       // shared, this warp's: pages of the group being copied
    uint8_t *live;      // and its live slots, a bit each
    Jobs jobs;
    int job_units, job_at;   // units of the newest group's job, and the first of this warp's without a group
    int units;               // of all jobs before that one
    Group now, mid, far;
    int id_mid[kEach], id_far[kEach];   // as they are in the table
    int pos_mid[8];
    int count;          // units copied (TMA), or the unit being copied
    bool over;          // no further job

    __device__ __forceinline__ Producer(const KvView &kv_, const AttendArgs &a_, const CUtensorMap *mk,
                                        const CUtensorMap *mv, Pipe<T, DP, NT> &pipe_, int per_seq_, const Jobs &j,
                                        char *smem_, int pw_)
        : kv(kv_), a(a_), map(pw_ ? mv : mk), pipe(pipe_), smem(smem_), per_seq(per_seq_), pw(pw_),
          lane(threadIdx.x & 31), us(S::kUnit / a_.hpu), per_tile(256 / (us / 16) + 1), jobs(j) {
        ids = reinterpret_cast<int32_t *>(smem + S::kRing + S::kMerge + pw * kLookup);
        live = reinterpret_cast<uint8_t *>(ids + 128);
        job_units = job_at = count = units = 0;
        over = false;
        now.units = mid.units = far.units = 0;
    }
    __device__ __forceinline__ uint32_t offset(int s) const { return (uint32_t)s - kv.page.div(s) * kv.page.d; }
    // Slot and head of the (first) row of the lane's look-up e.
    __device__ __forceinline__ int slot_of(const Group &g, int e, int &head) const {
        const int row = TMA ? 8 * lane : 32 * e + lane, u = row / S::kUnit, in = row - u * S::kUnit;
        head = head_of(in);
        return g.s + u * kTurn * us + in - head * us;
    }
    // Which of the unit's heads row `in` belongs to: its tile (below 8) over the tiles of a head.
    __device__ __forceinline__ int head_of(int in) const { return (in >> 4) * per_tile >> 8; }
    __device__ __forceinline__ bool is_page(int id) const { return (uint32_t)id < (uint64_t)kv.c.pages; }
    // The next group becomes `now`, its pages and live slots in shared memory.
    __device__ __forceinline__ void step() {
        __syncwarp();
        if (mid.units > 0) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                ids[32 * e + lane] = id_mid[e];
                if constexpr (TMA) {
                    int head;
                    uint32_t on = is_page(id_mid[0]) ? 0xffu >> max(0, 8 - (mid.end - slot_of(mid, 0, head))) : 0u;
                    if (a.first) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) on &= ~((uint32_t)(pos_mid[x] < mid.low) << x);
                    }
                    live[lane] = (uint8_t)on;
                } else {
                    const uint32_t on = __ballot_sync(0xffffffffu, is_page(id_mid[e]) && !(a.first && pos_mid[e] < mid.low));
                    if (lane == 0) reinterpret_cast<uint32_t *>(live)[e] = on;
                }
            }
        }
        now = mid, mid = far;
        __syncwarp();
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            id_mid[e] = id_far[e];
            if (!a.first || mid.units == 0 || !is_page(id_mid[e])) continue;
            int head;
            const uint32_t off = offset(slot_of(mid, e, head));
            const int32_t *p = kv.c.position + kv.mark(id_mid[e], mid.h + head, off);
            if constexpr (TMA) {   // 8 slots of a page whose size is a multiple of 8
                const int4 x = reinterpret_cast<const int4 *>(p)[0], y = reinterpret_cast<const int4 *>(p)[1];
                pos_mid[0] = x.x, pos_mid[1] = x.y, pos_mid[2] = x.z, pos_mid[3] = x.w;
                pos_mid[4] = y.x, pos_mid[5] = y.y, pos_mid[6] = y.z, pos_mid[7] = y.w;
            } else {
                pos_mid[e] = *p;
            }
        }
        far.units = 0;
        while (job_at >= job_units && !over) {   // a job may have no unit of this warp's
            units += job_units;
            if (!jobs.next(kv, a, us, per_seq)) over = true, job_units = 0;
            // A job without a slot (whole jobs only) is one unit without a live one.
            else job_units = max(1, jobs.b1 - jobs.b0);
            job_at = TMA ? 0 : (pw + units) & (kProducers - 1);
        }
        if (!over) {
            far.i = jobs.i, far.h = jobs.r / a.hb * a.hpu, far.hb = jobs.r % a.hb, far.end = jobs.last(us);
            far.s = jobs.first(us) + job_at * us;
            far.units = min(kUnits, (job_units - job_at + kTurn - 1) / kTurn);
            far.unit = job_at, far.of = job_units, far.base = units;
            far.low = a.first ? a.first[jobs.i] : 0;
            if (job_at == 0 && (!TMA || pw == 0)) {   // the queries come from memory by the time the job begins
                const int qh = far.h * a.group + far.hb * S::kHeads;
                const int words = min(S::kHeads, a.group * a.hpu - far.hb * S::kHeads) * kv.c.head_dim;
                const float *q = a.q + far.i * a.ldq + (int64_t)qh * kv.c.head_dim;
                for (int x = 32 * lane; x < words; x += 1024) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + x));
            }
            job_at += far.units * kTurn;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                int head;
                const int row = TMA ? 8 * lane : 32 * e + lane, s = slot_of(far, e, head);
                id_far[e] = -1;
                if (row < far.units * S::kUnit && s < far.end)   // checked when it is used, a group later
                    id_far[e] = kv.c.table[far.i * kv.c.ld_table + kv.page.div((uint32_t)s)];
            }
        }
    }
    // All units of the block; false when a bounded wait ran out.
    __device__ __forceinline__ bool run() {
        for (;;) {
            while (now.units == 0) {
                if (over && mid.units == 0 && far.units == 0) return true;
                step();
            }
            for (int u = 0; u < now.units; ++u) {
                const int s = now.s + u * kTurn * us, unit = now.unit + u * kTurn;
                // Lane k: the live slots of tile k.
                const uint32_t on = lane < kHalves ? reinterpret_cast<const uint16_t *>(live)[u * kHalves + lane] : 0;
                const uint32_t any = __ballot_sync(0xffffffffu, on != 0);
                const bool last = unit + 1 == now.of;
                if (TMA && !any && !last) continue;
                if (!TMA) count = now.base + unit;
                const int stage = count % S::kStages;
                if (count >= S::kStages &&
                    !mbar_wait(pipe.empty + stage, (count / S::kStages - 1) & 1, &pipe.aborted))
                    return false;
                __syncwarp();
                if (!TMA || pw == 0) {
                    if (lane < kHalves) pipe.live[stage][lane] = (uint16_t)on;
                    if (lane == 0) pipe.unit[stage] = unit | (last ? kLastUnit : 0);
                    __syncwarp();
                }
                if constexpr (TMA) {
                    if (a.box == 0) box_of_all(any != 0, u, s, stage);
                    else if (a.box == 8) boxes<8>(u, s, stage);
                    else if (a.box == 16) boxes<16>(u, s, stage);
                    else if (a.box == 32) boxes<32>(u, s, stage);
                    else boxes<64>(u, s, stage);
                } else {
                    rows(u, s, stage);
                }
                ++count;
            }
            now.units = 0;
        }
    }
    // The unit is one box (us slots of a page, of a.hpu heads).
    __device__ __forceinline__ void box_of_all(bool any, int u, int s, int stage) {
        if (lane == 0) {
            uint64_t *bar = pipe.full + stage;
            mbar_expect_tx(bar, any ? (uint32_t)(S::kUnit * S::kRow) : 0u);
            char *to = smem + stage * S::kStage + pw * (S::kStage / 2);
            const int page = ids[u * S::kUnit / 8];
            if (any) {
#pragma unroll
                for (int k = 0; k < S::kRow / 128; ++k)
                    tma_load_4d(to + k * 128 * S::kUnit, map, bar, k * 128 / S::kES, (int)offset(s), now.h, page);
            }
        }
        __syncwarp();
    }
    // Boxes of one head.  Straight code: a lane issues a copy in about 100
    // cycles, 200 in a loop over boxes.
    template <int BOX>
    __device__ __forceinline__ void boxes(int u, int s, int stage) {
        if constexpr (S::kUnit % BOX == 0) {
            constexpr int N = S::kUnit / BOX;
            const uint8_t *on = live + u * (S::kUnit / 8);
            bool has = false;
            if (lane < N) {
#pragma unroll
                for (int x = 0; x < BOX / 8; ++x) has |= on[lane * (BOX / 8) + x] != 0;
            }
            const uint32_t mask = __ballot_sync(0xffffffffu, has);
            if (lane == 0) {
                uint64_t *bar = pipe.full + stage;
                mbar_expect_tx(bar, (uint32_t)(__popc(mask) * BOX) * S::kRow);
                int page[N];
#pragma unroll
                for (int b = 0; b < N; ++b) page[b] = ids[(u * S::kUnit + b * BOX) / 8];
                char *to = smem + stage * S::kStage + pw * (S::kStage / 2);
                const int off0 = (int)offset(s);
                int off = off0, h = now.h, row = 0;
#pragma unroll
                for (int b = 0; b < N; ++b) {
                    if (mask >> b & 1u) {
                        const int c1 = a.token_major ? h : off, c2 = a.token_major ? off : h;
#pragma unroll
                        for (int k = 0; k < S::kRow / 128; ++k)
                            tma_load_4d(to + b * BOX * 128 + k * 128 * S::kUnit, map, bar, k * 128 / S::kES, c1, c2,
                                        page[b]);
                    }
                    off += BOX, row += BOX;
                    if (off == (int)kv.page.d) off = 0;
                    if (row == us) off = off0, ++h, row = 0;   // the next head's slots
                }
            }
            __syncwarp();
        }
    }
    __device__ __forceinline__ void rows(int u, int s, int stage) {
        const char *kp = static_cast<const char *>(kv.c.k), *vp = static_cast<const char *>(kv.c.v);
        const int chunks = kv.c.head_dim * S::kES / 16;
        const uint32_t to = smem_u32(smem + stage * S::kStage);
        for (int r0 = 0; r0 < S::kUnit; r0 += 32) {   // a lane's row: 16 or 32 of a head's
            const int in = r0 + lane, e = u * S::kUnit + in, head = head_of(in);
            const bool on = in < S::kUnit && live[e >> 3] >> (e & 7) & 1u;
            const int64_t row = on ? kv.element(ids[e], now.h + head, offset(s + in - head * us)) * S::kES : -1;
            const uint32_t any = __ballot_sync(0xffffffffu, on);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (!(any >> (16 * half) & 0xffffu)) continue;   // a tile without a live slot is not read
#pragma unroll 8
                for (int x = 0; x < 16 * S::kChunks / 32; ++x) {
                    const int at16 = x * 32 + lane, rr = 16 * half + at16 / S::kChunks, c = at16 % S::kChunks;
                    const int64_t from = __shfl_sync(0xffffffffu, row, rr);
                    const bool ok = from >= 0 && c < chunks;
                    const uint32_t dst = to + chunk_at<128 * S::kUnit>(r0 + rr, c);
                    const int64_t src = ok ? from + c * 16 : 0;
                    copy16(dst, kp + src, ok);
                    copy16(dst + S::kStage / 2, vp + src, ok);
                }
            }
        }
        copies_arrive(pipe.full + stage);
        if (lane == 0) mbar_arrive(pipe.full + stage);   // with the stage's live slots and unit
    }
    // Nothing in flight may outlive the block, should the consumers have given up.
    __device__ __forceinline__ void drain() {
        if constexpr (TMA) {
            for (int c = max(0, count - S::kStages); c < count; ++c)
                mbar_drain(pipe.full + c % S::kStages, c / S::kStages & 1);
        } else {
            copies_wait_all();
        }
    }
};

template <int THREADS>
__device__ __forceinline__ void consumers_sync() {
    asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

template <class T, int DP, int NT, bool TMA>
__global__ void __launch_bounds__(32 * (Shape<T, DP, NT>::kWarps + kProducers),
                                  Shape<T, DP, NT>::kBlocks)
    attend_kernel(KvView kv, AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
    using S = Shape<T, DP, NT>;
    constexpr int W = S::kWarps, P = kProducers, THREADS = 32 * W, ALL = THREADS + 32 * P, MS = S::kSlots;
    extern __shared__ __align__(1024) char smem[];
    static_assert(sizeof(Pipe<T, DP, NT>) <= S::kMisc, "pipe");
    Pipe<T, DP, NT> &pipe = *reinterpret_cast<Pipe<T, DP, NT> *>(smem + S::kMiscAt);
    float *mo = reinterpret_cast<float *>(smem + S::kRing), *mm = mo + MS * S::kHeads * S::kPitch,
          *ml = mm + MS * S::kHeads;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, g = lane >> 2, t = lane & 3;
    const int D = kv.c.head_dim, per_seq = kv.c.kv_heads / a.hpu * a.hb, us = S::kUnit / a.hpu;
    if (tid == 0) {
        pipe.aborted = 0;
        for (int x = 0; x < S::kStages; ++x) {
            mbar_init(pipe.full + x, TMA ? P : 32 + 1);
            mbar_init(pipe.empty + x, W);
        }
        mbar_init_fence();
    }
    __syncthreads();
    pdl_enter();

    Jobs jobs;
    int64_t total = 0, end = 0;
    if (a.whole) {
        jobs.i = blockIdx.x / per_seq, jobs.at = blockIdx.x % per_seq, jobs.left = 1;
    } else {
        find_place<ALL>(kv, a, us, per_seq, blockIdx.x, gridDim.x, total, end, jobs, pipe.place);
        // Sequences without a slot belong to nobody's units: their rows are shared out.
        for (int64_t i = blockIdx.x; i < kv.c.seqs; i += gridDim.x)
            if (kv.length(a.lens, i, a.max_len) == 0)
                for (int x = tid; x < a.heads * D; x += ALL) a.out[i * a.ldo + x] = 0.0f;
        if (tid == 0) a.split[3 * blockIdx.x] = -1;
    }
    if (w >= W) {
        Producer<T, DP, NT, TMA> producer(kv, a, &mk, &mv, pipe, per_seq, jobs, smem, w - W);
        if (!producer.run()) {
            *(volatile int *)&pipe.aborted = 1;   // results are void; the device status says so
            if (lane == 0) atomicExch(&g_attend_error, 1u);
        }
        producer.drain();
        return;
    }

    Warp<T, DP, NT> wp;
    int stage = 0, parity = 0;
    // The warp's head of a unit's, and which of the head's tiles of 16 slots.
    const int of_head = W / a.hpu, hi = w / of_head, sub = w - hi * of_head;
    uint32_t *qs = reinterpret_cast<uint32_t *>(smem + S::kQAt) + hi * S::kQWords;
    while (jobs.next(kv, a, us, per_seq)) {
        const int s0 = jobs.first(us), s1 = jobs.last(us);
        const int h = jobs.r / a.hb * a.hpu + hi, hb = jobs.r % a.hb;
        const int rows = min(S::kHeads, a.group - hb * S::kHeads);
        const int64_t i = jobs.i, qh = (int64_t)h * a.group + hb * S::kHeads;
        float *scores = a.scores ? a.scores + (i * a.heads + qh) * a.score_rows + s0 : nullptr;
        wp.clear();
        wp.queries(a.q + i * a.ldq + qh * D, D, rows, a.scale2, qs);
        if constexpr (!S::kQReg) consumers_sync<THREADS>();
        for (int n = max(1, jobs.b1 - jobs.b0); n > 0; --n) {   // at most; the job's last unit ends it
            if (!mbar_wait(pipe.full + stage, parity, &pipe.aborted)) {
                *(volatile int *)&pipe.aborted = 1;
                if (lane == 0) atomicExch(&g_attend_error, 1u);
                break;
            }
            const uint32_t live = pipe.live[stage][w];
            const int unit = pipe.unit[stage], at = (unit & (kLastUnit - 1)) * us + 16 * sub;
            char *k = smem + stage * S::kStage + 16 * w * 128, *v = k + S::kStage / 2;
            float *sc = scores && s0 + at < s1 ? scores + at : nullptr;   // rows of 16 slots exist in whole
            if (live) {
                if (live != 0xffffu) {   // a weight of zero does not make up for a NaN in a slot that does not count
                    for (int x = lane; x < 16 * S::kChunks; x += 32)
                        if (!(live >> (x / S::kChunks) & 1u))
                            *reinterpret_cast<uint4 *>(v + chunk_at<128 * S::kUnit>(x / S::kChunks, x % S::kChunks)) =
                                make_uint4(0, 0, 0, 0);
                    if (TMA) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before the next copy
                    __syncwarp();
                }
                wp.tile(smem_u32(k), smem_u32(v), live, qs, sc, a.score_rows, rows);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(pipe.empty + stage);
            if (++stage == S::kStages) stage = 0, parity ^= 1;
            if (unit & kLastUnit) break;
        }

        // Merge of a head's warps through shared memory, the uppermost into those
        // before them, and so on.
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) wp.l[n][j] += __shfl_xor_sync(0xffffffffu, wp.l[n][j], x);
                if constexpr (kScaleP<T> != 1.0f) {
                    wp.l[n][j] *= 1.0f / kScaleP<T>;
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) wp.o[n][x][j] *= 1.0f / kScaleP<T>, wp.o[n][x][2 + j] *= 1.0f / kScaleP<T>;
                }
            }
        auto put = [&](int slot) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int head = slot * S::kHeads + 8 * n + 2 * t + j;
                    if (8 * n + 2 * t + j >= rows) continue;
                    if (g == 0) mm[head] = wp.m[n][j], ml[head] = wp.l[n][j];
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        mo[head * S::kPitch + 16 * x + g] = wp.o[n][x][j];
                        mo[head * S::kPitch + 16 * x + g + 8] = wp.o[n][x][2 + j];
                    }
                }
        };
        auto take = [&](int slot) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int head = slot * S::kHeads + 8 * n + 2 * t + j;
                    if (8 * n + 2 * t + j >= rows) continue;
                    const float m = mm[head], top = fmaxf(m, wp.m[n][j]), ref = top == minus_inf() ? 0.0f : top;
                    const float f = power2(wp.m[n][j] - ref), e = power2(m - ref);
                    wp.m[n][j] = top;
                    wp.l[n][j] = fmaf(e, ml[head], f * wp.l[n][j]);
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        wp.o[n][x][j] = fmaf(e, mo[head * S::kPitch + 16 * x + g], f * wp.o[n][x][j]);
                        wp.o[n][x][2 + j] = fmaf(e, mo[head * S::kPitch + 16 * x + g + 8], f * wp.o[n][x][2 + j]);
                    }
                }
            __syncwarp();
        };
        const int buffers = max(1, MS / a.hpu);   // of a head; a.hpu <= MS where a head has several warps
        for (int top = of_head; top > 1;) {
            const int n = min(buffers, top / 2);
            const int taker = sub + n;   // whose result this warp takes; a warp's later put goes where it took from
            if (sub >= top - n && sub < top) put(hi * buffers + sub % buffers);
            consumers_sync<THREADS>();
            if (sub >= top - 2 * n && sub < top - n) take(hi * buffers + taker % buffers);
            top -= n;
        }
        const bool whole = jobs.b0 == 0 && jobs.b1 == jobs.nb;
        if (sub == 0) {
            const int64_t part = ((2 * (int64_t)blockIdx.x + (jobs.b0 == 0 ? 1 : 0)) * a.hpu + hi) * S::kHeads;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int head = 8 * n + 2 * t + j;
                    if (head >= rows) continue;
                    const float m = wp.m[n][j], sum = wp.l[n][j], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                    if (whole) {
                        float *out = a.out + i * a.ldo + (qh + head) * D;
#pragma unroll
                        for (int x = 0; x < DP / 16; ++x) {
                            // (an infinite value: as with keys)
                            if (16 * x + g < D) out[16 * x + g] = finite_or_nan(wp.o[n][x][j] * inv);
                            if (16 * x + g + 8 < D) out[16 * x + g + 8] = finite_or_nan(wp.o[n][x][2 + j] * inv);
                        }
                        if (a.scores && g == 0) {
                            const float ref = m == minus_inf() ? 0.0f : m;
                            if (a.whole && a.hb == 1) pipe.stats[hi * S::kHeads + head] = make_float2(ref, inv);
                            else *reinterpret_cast<float2 *>(a.stats + 2 * (i * a.heads + qh + head)) = make_float2(ref, inv);
                        }
                    } else {
                        float *out = a.part_o + (part + head) * DP;
#pragma unroll
                        for (int x = 0; x < DP / 16; ++x) out[16 * x + g] = wp.o[n][x][j], out[16 * x + g + 8] = wp.o[n][x][2 + j];
                        if (g == 0) a.part_ml[2 * (part + head)] = m, a.part_ml[2 * (part + head) + 1] = sum;
                    }
                }
        }
        if (a.scores && a.whole && a.hb == 1) {
            // The job's scores are this block's: its weights need no further launch.
            consumers_sync<THREADS>();
            for (int x = 4 * (32 * sub + lane); x < s1; x += 128 * of_head) {   // a lane four slots
                const bool quad = a.quads && x + 4 <= s1;
                int64_t at[4];
                __align__(16) float old[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (quad && j) {
                        at[j] = at[0] < 0 ? -1 : at[0] + j;
                        continue;
                    }
                    uint32_t off;
                    const int id = x + j < s1 ? kv.page_of(i, (uint32_t)(x + j), off) : -1;
                    at[j] = id < 0 ? -1 : kv.mark(id, h, off);
                }
                if (quad && at[0] >= 0) *reinterpret_cast<float4 *>(old) = *reinterpret_cast<const float4 *>(kv.c.weight + at[0]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!quad && at[j] >= 0) old[j] = kv.c.weight[at[j]];
#pragma unroll 8
                for (int r = 0; r < rows; ++r) {   // rows of 16 slots exist in whole
                    const float2 st = pipe.stats[hi * S::kHeads + r];
                    const float4 v = *reinterpret_cast<const float4 *>(scores + r * a.score_rows + x);
                    sum[0] = fmaf(power2(v.x - st.x), st.y, sum[0]);
                    sum[1] = fmaf(power2(v.y - st.x), st.y, sum[1]);
                    sum[2] = fmaf(power2(v.z - st.x), st.y, sum[2]);
                    sum[3] = fmaf(power2(v.w - st.x), st.y, sum[3]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // Slots below the bound gather nothing (and may have no score).
                    if (a.first && at[j] >= 0 && kv.c.position[at[j]] < a.first[i]) sum[j] = 0.0f;
                    old[j] = fmaf(old[j], a.decay, sum[j]);
                }
                if (quad && at[0] >= 0) *reinterpret_cast<float4 *>(kv.c.weight + at[0]) = *reinterpret_cast<const float4 *>(old);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!quad && at[j] >= 0) kv.c.weight[at[j]] = old[j];
            }
        }
        if (!whole && jobs.b0 == 0 && tid == 0) {   // this block's end cuts the job: who has the rest of it?
            // Counted unit u is block c's if total c / blocks <= u < total (c + 1) / blocks (rounded down).
            const int64_t last = end + (jobs.nb - jobs.b1) - 1, n = gridDim.x;
            int64_t c = last * n / total;
            while (total * (c + 1) / n <= last) ++c;
            while (total * c / n > last) --c;
            a.split[3 * blockIdx.x] = i * per_seq + jobs.r;
            a.split[3 * blockIdx.x + 1] = c;
            a.split[3 * blockIdx.x + 2] = total;
        }
        if (of_head > 1 || !S::kQReg) consumers_sync<THREADS>();   // buffers and queries are free again
    }
}

template <class T, int DP, int NT, bool TMA>
int resident() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    static std::atomic<unsigned long long> done{0};
    using S = Shape<T, DP, NT>;
    if (!ensure_smem_limit(done, attend_kernel<T, DP, NT, TMA>, S::kBytes, &dev)) return 0;
    std::atomic<int> &at = known[dev & 63];
    if ((n = at.load(std::memory_order_relaxed)) > 0) return n;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, attend_kernel<T, DP, NT, TMA>, 32 * (S::kWarps + kProducers), S::kBytes) !=
        cudaSuccess)
        return 0;
    n *= sm_count(dev);
    at.store(n, std::memory_order_relaxed);
    return n;
}

// A pool as a tensor of (channel, slot, head, page), or (channel, head, slot,
// page) where heads are the closer ones; box: 128 bytes of `slots_box` slots of
// `heads_box` heads.  False where the strides do not nest (the lanes copy), or
// for several heads where heads are the closer ones.
template <class T>
bool pool_map(CUtensorMap *map, const mosaic_kv_cache &c, void *pool, int slots_box, int heads_box, int *token_major) {
    constexpr int kES = sizeof(T);
    const cuuint64_t D = (cuuint64_t)c.head_dim * kES, slots = (cuuint64_t)c.page_size, heads = (cuuint64_t)c.kv_heads;
    cuuint64_t slot = (cuuint64_t)c.slot_stride * kES, head = (cuuint64_t)c.head_stride * kES;
    cuuint64_t page = (cuuint64_t)c.page_stride * kES;
    if (heads == 1) head = slot * slots;
    const bool tm = head < slot;
    if (tm && heads_box > 1) return false;
    const cuuint64_t inner = tm ? head : slot, outer = tm ? slot : head;
    if (c.pages == 1) page = outer * (tm ? slots : heads);
    const cuuint64_t most = (cuuint64_t)1 << 40;
    if (inner < D || outer < inner || page < outer || outer % inner || page % outer || page >= most) return false;
    auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, tm ? heads : slots, tm ? slots : heads, (cuuint64_t)c.pages};
    const cuuint64_t strides[3] = {inner, outer, page};
    const cuuint32_t box[4] = {128 / kES, tm ? 1u : (cuuint32_t)slots_box, tm ? (cuuint32_t)slots_box : (cuuint32_t)heads_box, 1}, each[4] = {1, 1, 1, 1};
    const CUtensorMapDataType type = kES == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : kTerms<T> == 3 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    *token_major = tm;
    return fn(map, type, 4, pool, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int DP, int NT>
struct Instance {
    using S = Shape<T, DP, NT>;
    // Heads share a unit if there is room for their queries, and a merge buffer or a warp for each.
    static AttendShape shape() {
        return {S::kHeads, DP, S::kUnit, S::kQReg ? S::kWarps : S::kQHeads, S::kSlots, S::kBlocks};
    }
    template <bool TMA>
    static mosaic_status go(const KvView &kv, AttendArgs a, const CUtensorMap &mk, const CUtensorMap &mv,
                            int &blocks, cudaStream_t st) {
        const int wave = resident<T, DP, NT, TMA>();
        if (wave <= 0) return MOSAIC_ERR_CUDA;
        if (!a.whole && a.blocks > wave) a.blocks = wave;
        blocks = a.blocks;
        {
            KernelSpan span("attend", st);
            const dim3 grid((unsigned)a.blocks), block(32 * (S::kWarps + kProducers));
            // More than one wave (whole jobs) must not stack up early.
            if (a.blocks <= wave) pdl_launch(attend_kernel<T, DP, NT, TMA>, grid, block, S::kBytes, st, kv, a, mk, mv);
            else attend_kernel<T, DP, NT, TMA><<<grid, block, S::kBytes, st>>>(kv, a, mk, mv);
        }
        return launch_status();
    }
    static mosaic_status launch(const mosaic_kv_cache &c, AttendArgs a, int &blocks, cudaStream_t st) {
        const KvView kv(c);
        alignas(64) CUtensorMap mk = {}, mv = {};
        // Positions are read 8 at a time.
        if (c.page_size % 8 == 0 && (!a.first || aligned16(c.position))) {
            const int us = S::kUnit / a.hpu;
            a.box = 0;   // a unit is one box
            if (us <= 64 && c.page_size % us == 0 && pool_map<T>(&mk, c, c.k, us, a.hpu, &a.token_major) &&
                pool_map<T>(&mv, c, c.v, us, a.hpu, &a.token_major) && (a.hpu > 1 || !a.token_major))
                return go<true>(kv, a, mk, mv, blocks, st);
            // As many slots of a head as divide a page and a unit, 8 at least (a swizzle's rows).
            for (a.box = 64; us % a.box || c.page_size % a.box; a.box /= 2) {
            }
            if (pool_map<T>(&mk, c, c.k, a.box, 1, &a.token_major) && pool_map<T>(&mv, c, c.v, a.box, 1, &a.token_major))
                return go<true>(kv, a, mk, mv, blocks, st);
        }
        return go<false>(kv, a, mk, mv, blocks, st);
    }
};

// The instance for a head_dim and a group: up to 8 query heads a tile, else 16.
template <class T, class F>
auto with_instance(int head_dim, int group, F f) {
    if (group <= 8) {
        if (head_dim <= 64) return f(Instance<T, 64, 1>());
        if (head_dim <= 128) return f(Instance<T, 128, 1>());
        return f(Instance<T, 256, 1>());
    }
    if (head_dim <= 64) return f(Instance<T, 64, 2>());
    if (head_dim <= 128) return f(Instance<T, 128, 2>());
    return f(Instance<T, 256, 2>());
}

}  // namespace

#define MOSAIC_ATTEND_TYPE(T)                                                                             \
    template <> AttendShape attend_shape<T>(int head_dim, int group) {                                    \
        return with_instance<T>(head_dim, group, [&](auto i) { return decltype(i)::shape(); });           \
    }                                                                                                     \
    template <>                                                                                           \
    mosaic_status attend_launch<T>(const mosaic_kv_cache &c, const AttendArgs &a, int &blocks,            \
                                   cudaStream_t st) {                                                     \
        return with_instance<T>(c.head_dim, a.group,                                                      \
                                [&](auto i) { return decltype(i)::launch(c, a, blocks, st); });           \
    }                                                                                                     \
    template <> mosaic_status attend_status<T>() {                                                        \
        unsigned int e = 0, zero = 0;                                                                     \
        if (cudaMemcpyFromSymbol(&e, g_attend_error, sizeof(e)) != cudaSuccess) return MOSAIC_ERR_CUDA;   \
        if (!e) return MOSAIC_OK;                                                                         \
        if (cudaMemcpyToSymbol(g_attend_error, &zero, sizeof(zero)) != cudaSuccess) return MOSAIC_ERR_CUDA; \
        return MOSAIC_ERR_TIMEOUT;                                                                        \
    }

}  // namespace mosaic
