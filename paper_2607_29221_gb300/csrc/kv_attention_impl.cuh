// The split kernel of kv_attention.cuh for one element type.
#pragma once

#include "kv_attention.cuh"

namespace mosaic {
namespace {

__device__ __forceinline__ uint32_t shared_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or zeros where !ok (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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
// d += a b, 16 x 8 x 16 (16-bit types) or 16 x 8 x 8 (tf32).
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3},{%4,%5,%6,%7},{%8,%9},{%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(__nv_bfloat16 x, __nv_bfloat16 y) {
    return __bfloat16_as_ushort(x) | (uint32_t)__bfloat16_as_ushort(y) << 16;
}
__device__ __forceinline__ uint32_t pack(__half x, __half y) {
    return __half_as_ushort(x) | (uint32_t)__half_as_ushort(y) << 16;
}

// x, y -> terms t[0] (the least) .. t[N-1] (the greatest), packed.
template <class T, int N>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        const T a = Elem<T>::from(x), b = Elem<T>::from(y);
        t[i] = pack(a, b);
        x -= Elem<T>::to(a), y -= Elem<T>::to(b);
    }
}
// fp32 as two tf32 terms, the upper one rounded to nearest (the lower one then
// has either sign, and what is left out averages out); the lower one's own tail
// (2^-23) is cut by the tensor core.
__device__ __forceinline__ uint32_t tf32_high(float x) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t tf32_low(float x, uint32_t high) {
    return __float_as_uint(x - __uint_as_float(high));
}

template <class T> constexpr int kTerms = sizeof(T) == 4 ? 2 : 3;
template <> constexpr int kTerms<__half> = 2;
// Probabilities are kept times 2^shift, so that fp16's lower term stays clear of subnormals.
template <class T> constexpr float kShift = 0.0f;
template <> constexpr float kShift<__half> = 12.0f;

// DP: head_dim padded to 64, 128 or 256.  NT: tiles of 8 query heads.
template <class T, int DP, int NT>
struct Shape {
    static constexpr int kES = sizeof(T), kRow = DP * kES, kChunks = kRow / 16;
    static constexpr int kTile = 2 * 16 * kRow;                   // K and V of 16 slots
    static constexpr int kWarps = kTile >= 32768 ? 2 : 4, kUnit = 16 * kWarps;
    static constexpr int kStages = kTile <= 4096 ? 4 : 3;
    static constexpr int kK = kES == 4 ? 8 : 16, kSteps = DP / kK;    // channels of a product step
    static constexpr int kHeads = 8 * NT, kPitch = DP + 4;
    static constexpr int kQWords = kSteps * NT * kTerms<T> * 2 * 32;  // query fragments
    // Queries stay in registers where they fit beside the outputs.
    static constexpr bool kQReg = kSteps * NT * kTerms<T> * 2 <= 48;
    static constexpr int kMerge = 4 * kWarps * kHeads * (kPitch + 2);
    static constexpr int kRing = kWarps * kStages * kTile;
    static constexpr int kQBytes = kQReg ? 0 : 4 * kQWords;
    static constexpr int kBytes = (kRing > kMerge ? kRing : kMerge) + kQBytes;
    static_assert(kBytes <= 227 * 1024, "shared memory");
};

// 16-byte chunk c of row r sits at chunk c ^ swizzle(r): 8 rows of a chunk are
// conflict-free (ldmatrix), and so are 8 words of 4 rows r, r + 1, r + 2, r + 3.
__device__ __forceinline__ int swizzle(int r) { return (r & 3) << 1 | (r >> 2 & 1); }

template <class T, int DP, int NT>
struct Warp {
    using S = Shape<T, DP, NT>;
    static constexpr int kTermsN = kTerms<T>;
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
            float mul = scale2;
            if constexpr (sizeof(T) == 2 && kTermsN == 2) {
                float top = 0.0f;
                for (int d = t; d < D; d += 4) top = fmaxf(top, in ? fabsf(x[d] * scale2) : 0.0f);
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // Largest |q| to [2^10, 2^11); nothing to scale in zeros, NaN and infinities.
                int e = (int)(__float_as_uint(top) >> 23) - 127;
                e = e == 128 || top == 0.0f ? 10 : e < -100 ? -100 : e;
                const float up = __uint_as_float((uint32_t)(10 - e + 127) << 23);
                const float down = __uint_as_float((uint32_t)(e - 10 + 127) << 23);
                mul = up;
                unscale[n][0] = __shfl_sync(0xffffffffu, down, 8 * t);
                unscale[n][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
            }
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k) {
                uint32_t f[kTermsN][2];
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int d = 8 * k + 4 * b + t;
                        const float v = in && d < D ? x[d] * scale2 : 0.0f;
                        f[1][b] = tf32_high(v);
                        f[0][b] = tf32_low(v, f[1][b]);
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int d = 16 * k + 8 * b + 2 * t;
                        float v = 0.0f, w = 0.0f;
                        if (in && d < D) v = x[d] * scale2, w = x[d + 1] * scale2;
                        if constexpr (kTermsN == 2) v *= mul, w *= mul;
                        uint32_t s[kTermsN];
                        split2<T, kTermsN>(v, w, s);
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

    // One tile of 16 slots, K rows at `tile` and V rows behind them; bit r of
    // `live`: slot r counts.  `sc`: where the scores of slot 0 go (rows of
    // `group` words, `heads` of which are the job's), or null; `left` rows exist.
    __device__ __forceinline__ void tile(uint32_t tile, uint32_t live, const uint32_t *qs, float *sc, int group,
                                         int heads, int left) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[n][j] = 0.0f;
        const int row = lane & 15, sw = swizzle(row & 7);   // swizzle depends on the row modulo 8
        const uint32_t base = tile + row * S::kRow;
#pragma unroll
        for (int k = 0; k < S::kSteps; ++k) {
            uint32_t a[4];
            ldm4(a, base + (((2 * k + (lane >> 4)) ^ sw) << 4));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (sizeof(T) == 4) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        hi[i] = tf32_high(__uint_as_float(a[i]));
                        lo[i] = tf32_low(__uint_as_float(a[i]), hi[i]);
                    }
                    mma(c, lo, query(qs, k, n, 1, 0), query(qs, k, n, 1, 1), T());
                    mma(c, hi, query(qs, k, n, 0, 0), query(qs, k, n, 0, 1), T());
                    mma(c, hi, query(qs, k, n, 1, 0), query(qs, k, n, 1, 1), T());
                } else {
#pragma unroll
                    for (int i = 0; i < kTermsN; ++i) mma(c, a, query(qs, k, n, i, 0), query(qs, k, n, i, 1), T());
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) s[n][j] += c[j];
            }
        }
        const bool up = live >> g & 1, dn = live >> (g + 8) & 1;
        uint32_t p16[NT][kTermsN][2];   // 16-bit types: terms of P^T, as the product wants them
        float alpha[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2 && kTermsN == 2) s[n][j] *= unscale[n][j & 1];
                s[n][j] = (j < 2 ? up : dn) ? s[n][j] : minus_inf();
            }
            if (sc) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = g + (j & 2) * 4, h = 8 * n + 2 * t + (j & 1);
                    if (r < left && h < heads) sc[(int64_t)r * group + h] = s[n][j];
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = fmaxf(s[n][j], s[n][2 + j]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                top = fmaxf(top, m[n][j]);
                alpha[n][j] = exp2f(m[n][j] - top);
                m[n][j] = top;
                const float ref = top - kShift<T>;
                s[n][j] = exp2f(s[n][j] - ref);
                s[n][2 + j] = exp2f(s[n][2 + j] - ref);
                l[n][j] = fmaf(l[n][j], alpha[n][j], s[n][j] + s[n][2 + j]);
            }
            if constexpr (sizeof(T) == 2) {
                uint32_t x[kTermsN], y[kTermsN];
                split2<T, kTermsN>(s[n][0], s[n][1], x);
                split2<T, kTermsN>(s[n][2], s[n][3], y);
#pragma unroll
                for (int i = 0; i < kTermsN; ++i) p16[n][i][0] = transpose8(x[i]), p16[n][i][1] = transpose8(y[i]);
            }
        }
        const uint32_t vbase = tile + 16 * S::kRow;
        if constexpr (sizeof(T) == 2) {
            // Slots (lane / 16) * 8 + lane % 8, channels 16 i + 8 (lane / 8 % 2).
            const int vr = (lane >> 4) * 8 + (lane & 7), vsw = swizzle(vr & 7);
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t a[4];
                ldm4t(a, vbase + vr * S::kRow + (((2 * i + (lane >> 3 & 1)) ^ vsw) << 4));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int x = 0; x < kTermsN; ++x) mma(c, a, p16[n][x][0], p16[n][x][1], T());
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][i][j] = fmaf(o[n][i][j], alpha[n][j & 1], c[j]);
                }
            }
        } else {
            uint32_t ph[NT][2][2], pl[NT][2][2];   // by step of 8 slots
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int from = (t + 4 * b) * 4 + (g >> 1);
                        const float x = __shfl_sync(0xffffffffu, s[n][2 * k], from);
                        const float y = __shfl_sync(0xffffffffu, s[n][2 * k + 1], from);
                        const float v = g & 1 ? y : x;
                        ph[n][k][b] = tf32_high(v);
                        pl[n][k][b] = tf32_low(v, ph[n][k][b]);
                    }
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                float c[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[n][j] = 0.0f;
                uint32_t hi[2][4], lo[2][4];
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = 8 * k + t + 2 * (j & 2), d = 16 * i + g + 8 * (j & 1);
                        const float v = lds(vbase + r * S::kRow + (((d >> 2) ^ swizzle(r & 7)) << 4) + (d & 3) * 4);
                        hi[k][j] = tf32_high(v);
                        lo[k][j] = tf32_low(v, hi[k][j]);
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        mma(c[n], lo[k], ph[n][k][0], ph[n][k][1], T());
                        mma(c[n], hi[k], pl[n][k][0], pl[n][k][1], T());
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) mma(c[n], hi[k], ph[n][k][0], ph[n][k][1], T());
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][i][j] = fmaf(o[n][i][j], alpha[n][j & 1], c[n][j]);
                }
            }
        }
    }
};

// The block's place in the row of all units.
struct Place {
    int64_t i;    // sequence
    int64_t at;   // units of it before the block's first
};

// Units of the whole call (`total`), and sequence and offset of unit `u0`.
// Every thread calls it; `sh` holds 2 x threads words.
template <int THREADS>
__device__ __forceinline__ void find_place(const KvView &kv, const AttendArgs &a, int unit, int64_t per_seq, int part,
                                           int parts, int64_t &total, int64_t &u0, int64_t &u1, Place &p,
                                           long long *sh) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t seqs = kv.c.seqs;
    auto units = [&](int64_t i) -> long long {
        return i < seqs ? (long long)((kv.length(a.lens, i, a.max_len) + unit - 1) / unit) * per_seq : 0;
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
    u0 = total * part / parts, u1 = total * (part + 1) / parts;
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
    p.i = sh[THREADS / 32], p.at = sh[THREADS / 32 + 1];
    __syncthreads();
}

template <class T, int DP, int NT>
__global__ void __launch_bounds__(32 * Shape<T, DP, NT>::kWarps) attend_kernel(KvView kv, AttendArgs a) {
    using S = Shape<T, DP, NT>;
    constexpr int W = S::kWarps, THREADS = 32 * W, NS = S::kStages;
    extern __shared__ __align__(1024) char smem[];
    __shared__ long long place_sh[W + 2];
    uint32_t *qs = reinterpret_cast<uint32_t *>(smem + S::kBytes - S::kQBytes);
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int D = kv.c.head_dim, KV = kv.c.kv_heads, per_seq = KV * a.hb;
    pdl_enter();

    int64_t u0, u1, total;
    Place p;
    if (a.whole) {
        p.i = blockIdx.x / per_seq;
        u0 = 0, u1 = 1, total = 0;
        p.at = 0;
    } else {
        find_place<THREADS>(kv, a, S::kUnit, per_seq, blockIdx.x, gridDim.x, total, u0, u1, p, place_sh);
        // Sequences without a slot belong to nobody's units: their rows are shared out.
        for (int64_t i = blockIdx.x; i < kv.c.seqs; i += gridDim.x)
            if (kv.length(a.lens, i, a.max_len) == 0)
                for (int x = tid; x < a.heads * D; x += THREADS) a.out[i * a.ldo + x] = 0.0f;
        if (tid == 0) a.split[3 * blockIdx.x] = -1;
    }

    const char *kp = static_cast<const char *>(kv.c.k), *vp = static_cast<const char *>(kv.c.v);
    const int chunks = D * S::kES / 16;
    const uint32_t ring = shared_addr(smem) + w * NS * S::kTile;
    Warp<T, DP, NT> wp;

    while (u0 < u1) {
        // The job of unit u0 and the block's slots [s0, s1) of it.
        const int len = kv.length(a.lens, p.i, a.max_len);
        const int nb = (len + S::kUnit - 1) / S::kUnit;
        int r, b0, b1;
        if (a.whole) {
            r = blockIdx.x % per_seq, b0 = 0, b1 = nb;
            u0 = u1;
        } else {
            if (nb == 0 || p.at >= (int64_t)nb * per_seq) {   // the next sequence
                p.i += 1, p.at = 0;
                continue;
            }
            r = (int)(p.at / nb), b0 = (int)(p.at - (int64_t)r * nb);
            const int64_t can = b0 + (u1 - u0);
            b1 = can < nb ? (int)can : nb;
            u0 += b1 - b0, p.at += b1 - b0;
        }
        const int h = r / a.hb, hb = r % a.hb;
        const int s0 = b0 * S::kUnit, s1 = min(len, b1 * S::kUnit);
        const int rows = min(S::kHeads, a.group - hb * S::kHeads);
        const int qh = h * a.group + hb * S::kHeads;
        wp.clear();
        const int low = a.first ? a.first[p.i] : 0;
        const int tiles = (s1 - s0 + 15) / 16, mine = tiles > w ? (tiles - w + W - 1) / W : 0;
        float *scores = a.scores ? a.scores + ((p.i * KV + h) * a.score_rows + s0) * a.group + hb * S::kHeads : nullptr;

        // Copies run NS - 1 tiles ahead, page ids one tile further, and with a
        // lower bound the positions in between.
        const int64_t nothing = -1;
        auto page_at = [&](int n, uint32_t &off) {
            const int s = s0 + 16 * (w + n * W) + (lane & 15);
            return n < mine && s < s1 ? kv.page_of(p.i, (uint32_t)s, off) : -1;
        };
        auto keep = [&](int id, uint32_t off) -> int64_t {   // element, or nothing if the slot is not live
            if (id < 0) return nothing;
            if (a.first && kv.c.position[kv.mark(id, h, off)] < low) return nothing;
            return kv.element(id, h, off) * S::kES;
        };
        uint32_t off_next = 0;
        int id_next = page_at(0, off_next);
        int64_t row_next = keep(id_next, off_next);
        id_next = page_at(1, off_next);
        unsigned long long queue = 0;
        auto issue = [&](int n, int depth) {
            const int64_t at = row_next;
            row_next = keep(id_next, off_next);
            id_next = page_at(n + 2, off_next);
            const uint32_t live = __ballot_sync(0xffffffffu, at >= 0) & 0xffffu;
            queue |= (unsigned long long)live << (16 * depth);
            if (live) {
                const uint32_t to = ring + (n % NS) * S::kTile;
#pragma unroll
                for (int x = 0; x < 16 * S::kChunks / 32; ++x) {
                    const int at16 = x * 32 + lane, rr = at16 / S::kChunks, c = at16 % S::kChunks;
                    const int64_t e = __shfl_sync(0xffffffffu, at, rr);
                    const bool ok = e >= 0 && c < chunks;
                    const uint32_t dst = to + rr * S::kRow + ((c ^ swizzle(rr & 7)) << 4);
                    const int64_t src = ok ? e + c * 16 : 0;
                    copy16(dst, kp + src, ok);
                    copy16(dst + 16 * S::kRow, vp + src, ok);
                }
            }
            copies_commit();
        };
#pragma unroll
        for (int n = 0; n < NS - 1; ++n) issue(n, n);
        wp.queries(a.q + p.i * a.ldq + (int64_t)qh * D, D, rows, a.scale2, qs);
        if constexpr (!S::kQReg) __syncthreads();
        for (int n = 0; n < mine; ++n) {
            copies_wait<NS - 2>();
            __syncwarp();
            const uint32_t live = (uint32_t)queue & 0xffffu;
            queue >>= 16;
            issue(n + NS - 1, NS - 2);
            const int s = 16 * (w + n * W);
            if (live)
                wp.tile(ring + (n % NS) * S::kTile, live, qs, scores ? scores + (int64_t)s * a.group : nullptr, a.group,
                        rows, s1 - s0 - s);
            else if (scores) {   // no slot counts: the weights read that
                for (int x = lane; x < 16 * rows; x += 32)
                    if (s + x / rows < s1 - s0) scores[(int64_t)(s + x / rows) * a.group + x % rows] = minus_inf();
            }
        }
        copies_wait<0>();

        // Merge of the warps.
        __syncthreads();
        float *mo = reinterpret_cast<float *>(smem), *mm = mo + W * S::kHeads * S::kPitch, *ml = mm + W * S::kHeads;
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float l = wp.l[n][j];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
                const int head = w * S::kHeads + 8 * n + 2 * t + j;
                if (g == 0) mm[head] = wp.m[n][j] - kShift<T>, ml[head] = l;
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    mo[head * S::kPitch + 16 * i + g] = wp.o[n][i][j];
                    mo[head * S::kPitch + 16 * i + g + 8] = wp.o[n][i][2 + j];
                }
            }
        __syncthreads();
        const bool whole = b0 == 0 && b1 == nb;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (b0 == 0 ? 1 : 0);
        for (int x = tid; x < rows * DP; x += THREADS) {
            const int head = x / DP, d = x % DP;
            float top = minus_inf(), sum = 0.0f, out = 0.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) top = fmaxf(top, mm[k * S::kHeads + head]);
            const float ref = top == minus_inf() ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const float f = exp2f(mm[k * S::kHeads + head] - ref);
                sum = fmaf(f, ml[k * S::kHeads + head], sum);
                out = fmaf(f, mo[(k * S::kHeads + head) * S::kPitch + d], out);
            }
            if (whole) {
                if (d < D) a.out[p.i * a.ldo + (int64_t)(qh + head) * D + d] = sum == 0.0f ? 0.0f : out / sum;
                if (a.scores && d == 0) {
                    float *st = a.stats + 2 * (p.i * a.heads + qh + head);
                    st[0] = ref, st[1] = sum;
                }
            } else {
                a.part_o[(slot * S::kHeads + head) * DP + d] = out;
                if (d == 0) a.part_ml[2 * (slot * S::kHeads + head)] = top, a.part_ml[2 * (slot * S::kHeads + head) + 1] = sum;
            }
        }
        if (!whole && b0 == 0 && tid == 0) {   // this block's end cuts the job: who else has a part of it?
            // Unit u is block c's if total c / blocks <= u < total (c + 1) / blocks (rounded down).
            const int64_t last = u1 + (nb - b1) - 1, n = gridDim.x;
            int64_t c = last * n / total;
            while (total * (c + 1) / n <= last) ++c;
            while (total * c / n > last) --c;
            a.split[3 * blockIdx.x] = p.i * per_seq + r;
            a.split[3 * blockIdx.x + 1] = c;
            a.split[3 * blockIdx.x + 2] = total;
        }
        __syncthreads();
    }
}

template <class T, int DP, int NT>
int resident() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    static std::atomic<unsigned long long> done{0};
    using S = Shape<T, DP, NT>;
    if (!ensure_smem_limit(done, attend_kernel<T, DP, NT>, S::kBytes, &dev)) return 0;
    std::atomic<int> &at = known[dev & 63];
    if ((n = at.load(std::memory_order_relaxed)) > 0) return n;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, attend_kernel<T, DP, NT>, 32 * S::kWarps, S::kBytes) !=
        cudaSuccess)
        return 0;
    n *= sm_count(dev);
    at.store(n, std::memory_order_relaxed);
    return n;
}

template <class T, int DP, int NT>
struct Instance {
    using S = Shape<T, DP, NT>;
    static AttendShape shape() { return {S::kHeads, DP, S::kUnit}; }
    static int wave() { return resident<T, DP, NT>(); }
    static mosaic_status launch(const mosaic_kv_cache &c, const AttendArgs &a, cudaStream_t st) {
        if (resident<T, DP, NT>() == 0) return MOSAIC_ERR_CUDA;   // sets the shared-memory limit
        const KvView kv(c);
        {
            KernelSpan span("attend", st);
            const dim3 grid((unsigned)a.blocks), block(32 * S::kWarps);
            // More than one wave (whole jobs) must not stack up early.
            if (a.blocks <= resident<T, DP, NT>())
                pdl_launch(attend_kernel<T, DP, NT>, grid, block, S::kBytes, st, kv, a);
            else attend_kernel<T, DP, NT><<<grid, block, S::kBytes, st>>>(kv, a);
        }
        return launch_status();
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

#define MOSAIC_ATTEND_TYPE(T)                                                                         \
    template <> AttendShape attend_shape<T>(int head_dim, int group) {                                \
        return with_instance<T>(head_dim, group, [&](auto i) { return decltype(i)::shape(); });       \
    }                                                                                                 \
    template <> int attend_wave<T>(int head_dim, int group) {                                         \
        return with_instance<T>(head_dim, group, [&](auto i) { return decltype(i)::wave(); });        \
    }                                                                                                 \
    template <>                                                                                       \
    mosaic_status attend_launch<T>(const mosaic_kv_cache &c, const AttendArgs &a, cudaStream_t st) {  \
        return with_instance<T>(c.head_dim, a.group, [&](auto i) { return decltype(i)::launch(c, a, st); }); \
    }

}  // namespace mosaic
