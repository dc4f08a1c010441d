// Attention of one new token per sequence over a 4-bit cache: the split, the
// producers and the join of kv_attention.cuh with consumer warps of its own.
//
// Bound by issuing instructions: a tile of 16 slots of 128 channels is 2560
// bytes, 109 cycles of an SM at HBM's rate, and takes 440 warp instructions, 208
// of which make fp16 values of its 4-bit codes (13 for 8, shared by all query
// heads).  Masks and fp16 arithmetic issue every second cycle a scheduler, and
// they and mma.sync (8 cycles) overlap little: 170 to 185 cycles.  (64 x 16384
// slots: 194 us, 141 without the conversion, 162 without the products.)  So
// everything else is arranged to need few:
//
//  * S = Q K^T and O += P V on mma.sync with K and V as the narrow operand (8
//    slots, 8 channels): 16 rows are 8 query heads twice, the upper and the lower
//    fp16 term of each query and probability, so one product has both, and P
//    goes from the first product's result to the second's operand without a move.
//  * Channels may be numbered at will in both products, as long as Q and O are
//    numbered alike: a lane's share of a row is 16 bytes (K) or 8 (V) in a piece,
//    one or two 128-bit loads, with a single step and base; two rows of V become
//    pairs of slots by one byte permutation a word.
//  * 32 slots a warp at a time: the softmax, the rescaling of O and the queries'
//    fragments (in shared memory) are shared by two tiles.  (64 at a time: 48
//    instructions fewer a tile, but twice the code: 208 -> 242 us.)
//
// Terms: queries are scaled to [2^14, 2^15) a head, probabilities by 2^15, and
// each is split into two fp16 numbers, 22 bits or 2^-25 of the scale: smaller
// query channels are off by up to 2^-39 of the head's largest, smaller weights
// by up to 2^-40 of the row's largest.  The 2^15 lies in the maximum that
// scores are taken off, lowered by 15 and rounded up, and so the same number
// for sums, outputs and joins at any score: probabilities reach 2^15 and never
// more (from scores of 2^24 on, whose steps are 2 and more, some bits less).  Products are exact in fp32; chains of
// four or two steps are added to the rest in fp32 with rounding to nearest, since
// the tensor cores truncate.
//
// Measured (device time): 131071 slots of 8 heads of 128 59 us with the join; 64
// sequences of up to 16384 195 (3.2 TB/s), 48 of up to 2000 on 32 heads 81.
#include "kv_attention_impl.cuh"

namespace mosaic {
namespace {

// TMA: copies by tensor boxes, else by lanes, which takes more warps: two / four,
// us, caches flushed, pages of 20.  400 sequences of up to 1500 on 8 key/value
// heads, bound 512: heads of 64 105 / 74, of 128 128 / 103; without a bound 111
// / 99, 149 / 151.  8 query heads each of 128, 48 of up to 2000: 63 / 65, 16 of
// up to 8000: 56 / 58.  (Four leave 128 registers, and heads of 128 spill 100 bytes.)
template <bool TMA>
struct Packed {};

template <bool TMA, int DP, int NT>
struct Shape<Packed<TMA>, DP, NT> {
    static constexpr int kES = 1, kRow = (5 * DP / 8 + 15) / 16 * 16, kChunks = kRow / 16;
    static constexpr int kProducers = TMA || DP * NT > 128 ? 2 : 4;
    static constexpr int kWarps = 4, kT = 2;   // kT: tiles of 16 slots that a warp takes at a time
    static constexpr int kUnit = 16 * kT * kWarps, kStage = 2 * kUnit * kRow;
    static constexpr int kStages = !TMA && DP * NT <= 128 ? 4 : DP * NT <= 128 ? 3 : 2;
    static constexpr int kSlots = 2;
    static constexpr int kSteps = DP / 16, kHeads = 8 * NT, kPitch = DP + 4;
    static constexpr int kQWords = kSteps * NT * 4 * 32;
    static constexpr bool kQReg = false;
    static constexpr int kQHeads = DP * NT <= 128 ? 4 : DP * NT == 256 ? 2 : 1;
    static constexpr int kRing = kStages * kStage, kMerge = 4 * kSlots * kHeads * (kPitch + 2), kIds = kProducers * kLookup<kUnit>;
    static constexpr int kQAt = (kRing + kMerge + kIds + 15) / 16 * 16, kMiscAt = kQAt + 4 * kQWords * kQHeads;
    static constexpr int kMisc = 512 + 8 * kHeads * kQHeads, kBytes = kMiscAt + kMisc;
    static constexpr int kPieces = 1, kPiece = kRow, kTiles = kUnit / 16;
    static constexpr bool kParted = true;
    static __device__ __forceinline__ uint32_t at(int r, int c) { return (uint32_t)(r * kRow + 16 * c); }
    static constexpr int kFit = 228 * 1024 / (kBytes + 1024), kMost = TMA && DP * NT <= 64 ? 3 : DP * NT <= 256 ? 2 : 1;
    static constexpr int kBlocks = kFit < kMost ? kFit : kMost;
    static_assert(kBytes <= 227 * 1024 && kBlocks >= 1, "shared memory");
};

__device__ __forceinline__ void lds4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
// N words in a row.
template <int N>
__device__ __forceinline__ void lds_words(uint32_t *r, uint32_t a) {
    if constexpr (N == 1) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[0]) : "r"(a) : "memory");
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(a) : "memory");
    else
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]) : "r"(a + 4 * i) : "memory");
}

template <bool TMA, int DP, int NT>
struct Warp4 {
    using S = Shape<Packed<TMA>, DP, NT>;
    // Words of codes of a lane: of a key row (channels DP / 4 t on), of a value row (DP / 8 g on); groups of the former.
    static constexpr int kT = S::kT, kKW = DP / 32, kVW = DP / 64, kKG = DP == 256 ? 2 : 1, kN = DP / 8;
    // Of head g; channels DP / 8 (2t + j) + i.  m: the largest score so far less 15, rounded up; l, o and what is made of
    // them (partial sums, statistics) are relative to it.
    float m[NT], l[NT], unscale[NT], o[NT][kN][2];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = minus_inf(), l[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < kN; ++i) o[n][i][0] = o[n][i][1] = 0.0f;
        }
    }
    // The job's queries as fragments in shared memory (step 2w + e of a lane has its
    // channels 8w + 2e, + 4 and 8w + 2e + 1, + 4, as q4_values gives them), and what
    // undoes their scaling.  Warp `sub` of `warps` takes every so many-th row, a
    // lane four neighbouring channels: rows come as whole lines (a lane that
    // fetched its own fragment's channels waited 15000 cycles, with all SMs at the
    // same lines).  Rows from `rows` to `last` become zeros, and those after them are.
    static __device__ __forceinline__ void queries(const float *q, int D, int rows, int last, float scale2, bool quads,
                                                   uint4 *qs, float2 *unscale, int sub, int warps) {
        constexpr int kParts = (DP + 127) / 128, kAtOnce = 4;   // rows in flight
        const int lane = threadIdx.x & 31;
        __half *const to = reinterpret_cast<__half *>(qs);
        for (int r0 = sub; r0 < last; r0 += kAtOnce * warps) {
            float v[kAtOnce][kParts][4];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x)
#pragma unroll
                for (int y = 0; y < kParts; ++y) {
                    const int r = r0 + x * warps, d = 128 * y + 4 * lane;
                    const float *from = q + (int64_t)r * D + d;
                    float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (r < rows && d < D) {   // multiples of four
                        if (quads) z = *reinterpret_cast<const float4 *>(from);
                        else z = make_float4(from[0], from[1], from[2], from[3]);
                    }
                    v[x][y][0] = z.x * scale2, v[x][y][1] = z.y * scale2, v[x][y][2] = z.z * scale2, v[x][y][3] = z.w * scale2;
                }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int r = r0 + x * warps, n = r >> 3, g = r & 7;
                if (r >= last) break;
                float top = 0.0f;
#pragma unroll
                for (int y = 0; y < kParts; ++y)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(v[x][y][i]));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                // Largest |q| to [2^14, 2^15); nothing to scale in zeros, NaN and infinities.
                int e = (int)(__float_as_uint(top) >> 23) - 127;
                e = e == 128 || top == 0.0f ? 14 : e < -100 ? -100 : e;
                const float up = __uint_as_float((uint32_t)(14 - e + 127) << 23);
                if (lane == 0) unscale[r].x = __uint_as_float((uint32_t)(e - 14 + 127) << 23);
#pragma unroll
                for (int y = 0; y < kParts; ++y) {
                    const int d = 128 * y + 4 * lane, t = d / (DP / 4), in = d % (DP / 4), half = in >> 2 & 1;
                    if (d >= DP) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {   // channel in + i: step 2 (in / 8) + i / 2, pair i % 2
                        const float z = v[x][y][i] * up;
                        const __half hi = __float2half_rn(z), lo = __float2half_rn(z - __half2float(hi));
                        __half *f = to + (((2 * (in >> 3) + (i >> 1)) * NT + n) * 32 + 4 * g + t) * 8 + (i & 1) * 4 + half;
                        f[0] = hi, f[2] = lo;
                    }
                }
            }
        }
    }

    // kT tiles of 16 slots, keys at k[], values at v[]; bit r of `live`: slot r
    // counts (kMasked: not all of them).  `sc`: where the scores of the tiles' first slots and
    // the job's first head go (a row of `pitch` words a head), or null.
    template <bool kMasked>
    __device__ __forceinline__ void tile(const uint32_t (&k)[kT], const uint32_t (&v)[kT], uint32_t live, uint32_t qs,
                                         float *const (&sc)[kT], int64_t pitch, int heads, int D) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float s[NT][4][2];   // 2t and 2t + 1 of 8 slots
        {
            uint32_t code[4][kKW], scale[4][kKG];
            const int scales = D / 2, groups = D / kQ4Group, g0 = DP == 64 ? t >> 1 : kKG * t;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t row = k[x >> 1] + ((x & 1) * 8 + g) * S::kRow;
                lds_words<kKW>(code[x], row + DP / 8 * t);
#pragma unroll
                for (int i = 0; i < kKG; ++i) {
                    lds_words<1>(&scale[x][i], row + scales + 4 * min(g0 + i, groups - 1));
                    if (g0 + i >= groups || (kMasked && !(live >> (8 * x + g) & 1u))) scale[x][i] = 0;
                }
            }
            constexpr int KB = S::kSteps < 4 ? S::kSteps : 4;   // steps of a chain
#pragma unroll
            for (int k0 = 0; k0 < S::kSteps; k0 += KB) {
                float c[4][NT][4];
#pragma unroll
                for (int w = 0; w < KB / 2; ++w) {
                    uint32_t a[2][NT][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int n = 0; n < NT; ++n) lds4(a[e][n], qs + (((k0 + 2 * w + e) * NT + n) * 32 + lane) * 16);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const __half2 sb = as_half2(scale[x][(k0 / 2 + w) / 4 % kKG]);
                        uint32_t y[4];
                        q4_values(code[x][k0 / 2 + w], __low2half2(sb), __high2half2(sb), y);
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if (w == 0 && e == 0) mma0(c[x][n], a[e][n], y[2 * e], y[2 * e + 1], __half());
                                else mma(c[x][n], a[e][n], y[2 * e], y[2 * e + 1], __half());
                            }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float z = c[x][n][j] + c[x][n][2 + j];
                            s[n][x][j] = k0 ? s[n][x][j] + z : z;
                        }
            }
        }
        uint32_t p[NT][kT][4];
        float alpha[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float most = 0.0f;   // an infinite score counts as NaN, also if only its scale makes it one
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int j = 0; j < 2; ++j) most = fmaxf(most, fabsf(s[n][x][j]));
            if (__any_sync(0xffffffffu, most * unscale[n] == __int_as_float(0x7f800000))) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[n][x][j] = fabsf(s[n][x][j] * unscale[n]) < __int_as_float(0x7f800000) ? s[n][x][j] : __int_as_float(0x7fffffff);
            }
            if constexpr (kMasked) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (!(live >> (8 * x + 2 * t + j) & 1u)) s[n][x][j] = minus_inf();
            }
            if (8 * n + g < heads) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (sc[x >> 1])
                        *reinterpret_cast<float2 *>(sc[x >> 1] + (8 * n + g) * pitch + (x & 1) * 8 + 2 * t) =
                            make_float2(s[n][x][0] * unscale[n], s[n][x][1] * unscale[n]);
            }
            float top = fmaxf(s[n][0][0], s[n][0][1]);
#pragma unroll
            for (int x = 1; x < 4; ++x) top = fmaxf(top, fmaxf(s[n][x][0], s[n][x][1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            top = fmaxf(m[n], __fadd_ru(top * unscale[n], -15.0f));
            alpha[n] = power2(m[n] - top);
            m[n] = top;
            float sum = 0.0f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float p0 = power2(fmaf(s[n][x][0], unscale[n], -top)), p1 = power2(fmaf(s[n][x][1], unscale[n], -top));
                sum += p0 + p1;
                const uint32_t hi = pack2(p0, p1, __half());
                const float2 r = unpack2(hi, __half());
                p[n][x >> 1][2 * (x & 1)] = hi;
                p[n][x >> 1][2 * (x & 1) + 1] = pack2(p0 - r.x, p1 - r.y, __half());
            }
            l[n] = fmaf(l[n], alpha[n], sum);
        }
        __half2 step[kT][2], base[kT][2];   // of slots 2t, 2t + 1 and 2t + 8, 2t + 9 of a tile
        const int gv = DP == 64 ? g >> 2 : DP == 128 ? g >> 1 : g, groups = D / kQ4Group, scales = D / 2 + 4 * min(gv, groups - 1);
#pragma unroll
        for (int y = 0; y < kT; ++y)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                uint32_t sb[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = 8 * b + 2 * t + j;
                    lds_words<1>(&sb[j], v[y] + r * S::kRow + scales);
                    if (gv >= groups || (kMasked && !(live >> (16 * y + r) & 1u))) sb[j] = 0;
                }
                step[y][b] = as_half2(__byte_perm(sb[0], sb[1], 0x5410));
                base[y][b] = as_half2(__byte_perm(sb[0], sb[1], 0x7632));
            }
        {
            uint32_t code[kT][4][kVW];
#pragma unroll
            for (int y = 0; y < kT; ++y)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    lds_words<kVW>(code[y][r], v[y] + (8 * (r >> 1) + 2 * t + (r & 1)) * S::kRow + DP / 16 * g);
#pragma unroll
            for (int i0 = 0; i0 < kN; i0 += 4) {   // half a word: four channels
                float c[4][NT][4];
#pragma unroll
                for (int y = 0; y < kT; ++y) {
                    uint32_t f[2][4];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        q4_values(__byte_perm(code[y][2 * b][i0 / 8], code[y][2 * b + 1][i0 / 8], i0 % 8 ? 0x7632 : 0x5410),
                                  step[y][b], base[y][b], f[b]);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (y == 0) mma0(c[x][n], p[n][y], f[0][x], f[1][x], __half());
                            else mma(c[x][n], p[n][y], f[0][x], f[1][x], __half());
                        }
                }
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float &to = o[n][i0 + x][j];
                            to = fmaf(to, alpha[n], c[x][n][j] + c[x][n][2 + j]);
                        }
            }
        }
    }
};

template <int DP, int NT, bool TMA>
__global__ void __launch_bounds__(32 * (Shape<Packed<TMA>, DP, NT>::kWarps + Shape<Packed<TMA>, DP, NT>::kProducers),
                                  Shape<Packed<TMA>, DP, NT>::kBlocks)
    attend4_kernel(KvView kv, AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
    using S = Shape<Packed<TMA>, DP, NT>;
    using P = Pipe<Packed<TMA>, DP, NT>;
    constexpr int W = S::kWarps, THREADS = 32 * W, ALL = THREADS + 32 * S::kProducers, MS = S::kSlots, kN = DP / 8, kT = S::kT;
    extern __shared__ __align__(1024) char smem[];
    static_assert(sizeof(P) <= S::kMisc, "pipe");
    P &pipe = *reinterpret_cast<P *>(smem + S::kMiscAt);
    float *mo = reinterpret_cast<float *>(smem + S::kRing), *mm = mo + MS * S::kHeads * S::kPitch, *ml = mm + MS * S::kHeads;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, g = lane >> 2, t = lane & 3;
    const int D = kv.c.head_dim, per_seq = kv.c.kv_heads / a.hpu * a.hb, us = S::kUnit / a.hpu;
    if (tid == 0) {
        pipe.aborted = 0;
        for (int x = 0; x < S::kStages; ++x) {
            mbar_init(pipe.full + x, TMA ? S::kProducers : 32 + 1);
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
            if (kv.length(a.lens, i, a.max_len) == 0) {
                for (int x = tid; x < a.heads * D; x += ALL) a.out[i * a.ldo + x] = 0.0f;
                if (a.by_job)
                    for (int r = tid; r < per_seq; r += ALL) a.split[3 * (i * per_seq + r)] = -1;
            }
        if (!a.by_job && tid == 0) a.split[3 * blockIdx.x] = -1;
    }
    if (w >= W) {
        Producer<Packed<TMA>, DP, NT, TMA> producer(kv, a, &mk, &mv, pipe, per_seq, jobs, smem, w - W);
        if (!producer.run()) {
            *(volatile int *)&pipe.aborted = 1;   // results are void; the device status says so
            if (lane == 0) atomicExch(&g_attend_error, 1u);
        }
        producer.drain();
        return;
    }

    Warp4<TMA, DP, NT> wp;
    int stage = 0, parity = 0;
    // The warp's head of a unit's, and which kT of the head's tiles of 16 slots.
    const int of_head = W / a.hpu, hi = w / of_head, sub = w - hi * of_head;
    uint4 *qs = reinterpret_cast<uint4 *>(smem + S::kQAt) + hi * (S::kQWords / 4);
    const int tile0 = kT * sub * a.hpu + hi;   // tiles of a head are a.hpu apart
    int held = 0;   // rows of the queries' fragments that are no zeros
    for (int x = 32 * sub + lane; x < S::kQWords / 4; x += 32 * of_head) qs[x] = make_uint4(0, 0, 0, 0);
    consumers_sync<THREADS>();
    while (jobs.next(kv, a, us, per_seq)) {
        const int s0 = jobs.first(us), s1 = jobs.last(us);
        const int h = jobs.r / a.hb * a.hpu + hi, hb = jobs.r % a.hb;
        const int rows = min(S::kHeads, a.group - hb * S::kHeads);
        const int64_t i = jobs.i, qh = (int64_t)h * a.group + hb * S::kHeads;
        float *scores = a.scores ? a.scores + (i * a.heads + qh) * a.score_rows + s0 : nullptr;
        wp.clear();
        float2 *stats = pipe.stats + hi * S::kHeads;   // in the end: maxima and sums
        wp.queries(a.q + i * a.ldq + qh * D, D, rows, max(rows, held), a.scale2, a.q_quads, qs, stats, sub, of_head);
        held = rows;
        consumers_sync<THREADS>();
#pragma unroll
        for (int n = 0; n < NT; ++n) wp.unscale[n] = 8 * n + g < rows ? stats[8 * n + g].x : 1.0f;
        for (int n = max(1, jobs.b1 - jobs.b0); n > 0; --n) {   // at most; the job's last unit ends it
            if (!mbar_wait(pipe.full + stage, parity, &pipe.aborted)) {
                *(volatile int *)&pipe.aborted = 1;
                if (lane == 0) atomicExch(&g_attend_error, 1u);
                break;
            }
            uint32_t live = 0;
#pragma unroll
            for (int x = 0; x < kT; ++x) live |= (uint32_t)pipe.live[stage][tile0 + x * a.hpu] << (16 * x);
            const int unit = pipe.unit[stage], at = (unit & (kLastUnit - 1)) * us + 16 * kT * sub;
            if (live) {
                const uint32_t base = smem_u32(smem + stage * S::kStage) + tile0 * 16 * S::kRow;
                uint32_t k[kT], v[kT];
                float *sc[kT];   // rows of 16 slots exist in whole
#pragma unroll
                for (int x = 0; x < kT; ++x) {
                    k[x] = base + x * a.hpu * 16 * S::kRow, v[x] = k[x] + S::kStage / 2;
                    sc[x] = scores && s0 + at + 16 * x < s1 ? scores + at + 16 * x : nullptr;
                }
                if (live == 0xffffffffu) wp.template tile<false>(k, v, live, smem_u32(qs), sc, a.score_rows, rows, D);
                else wp.template tile<true>(k, v, live, smem_u32(qs), sc, a.score_rows, rows, D);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(pipe.empty + stage);
            if (++stage == S::kStages) stage = 0, parity ^= 1;
            if (unit & kLastUnit) break;
        }

        // Merge of a head's warps through shared memory, the uppermost into those
        // before them, and so on.
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            wp.l[n] += __shfl_xor_sync(0xffffffffu, wp.l[n], 1);
            wp.l[n] += __shfl_xor_sync(0xffffffffu, wp.l[n], 2);
        }
        auto put = [&](int slot) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int head = slot * S::kHeads + 8 * n + g;
                if (8 * n + g >= rows) continue;
                if (t == 0) mm[head] = wp.m[n], ml[head] = wp.l[n];
#pragma unroll
                for (int x = 0; x < kN; ++x)
                    *reinterpret_cast<float2 *>(mo + head * S::kPitch + 8 * x + 2 * t) = make_float2(wp.o[n][x][0], wp.o[n][x][1]);
            }
        };
        auto take = [&](int slot) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int head = slot * S::kHeads + 8 * n + g;
                if (8 * n + g >= rows) continue;
                const float m = mm[head], top = fmaxf(m, wp.m[n]), ref = top == minus_inf() ? 0.0f : top;
                const float f = power2(wp.m[n] - ref), e = power2(m - ref);
                wp.m[n] = top;
                wp.l[n] = fmaf(e, ml[head], f * wp.l[n]);
#pragma unroll
                for (int x = 0; x < kN; ++x) {
                    const float2 y = *reinterpret_cast<const float2 *>(mo + head * S::kPitch + 8 * x + 2 * t);
                    wp.o[n][x][0] = fmaf(e, y.x, f * wp.o[n][x][0]);
                    wp.o[n][x][1] = fmaf(e, y.y, f * wp.o[n][x][1]);
                }
            }
            __syncwarp();
        };
        const int buffers = max(1, MS / a.hpu);   // of a head; a.hpu <= MS where a head has several warps
        // (of a single unit, those that had a slot)
        const int full = jobs.b1 - jobs.b0 > 1 ? of_head : min(of_head, max(1, (s1 - s0 + 16 * kT - 1) / (16 * kT)));
        for (int top = full; top > 1;) {
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
            for (int n = 0; n < NT; ++n) {
                const int head = 8 * n + g;
                if (head >= rows) continue;
                const float m = wp.m[n], sum = wp.l[n], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                float *out = whole ? a.out + i * a.ldo + (qh + head) * D : a.part_o + (part + head) * DP;
                const bool quads = !whole || a.out_quads;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int x = 0; x < kN; x += 4) {
                        const int d = kN * (2 * t + j) + x;
                        float y[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) y[z] = whole ? finite_or_nan(wp.o[n][x + z][j] * inv) : wp.o[n][x + z][j];
                        if (whole && d >= D) continue;
                        if (quads) *reinterpret_cast<float4 *>(out + d) = make_float4(y[0], y[1], y[2], y[3]);
                        else out[d] = y[0], out[d + 1] = y[1], out[d + 2] = y[2], out[d + 3] = y[3];
                    }
                if (t) continue;
                if (!whole) {
                    a.part_ml[2 * (part + head)] = m, a.part_ml[2 * (part + head) + 1] = sum;
                } else if (a.scores) {
                    const float ref = m == minus_inf() ? 0.0f : m;
                    if (a.whole && a.hb == 1) stats[head] = make_float2(ref, inv);
                    else *reinterpret_cast<float2 *>(a.stats + 2 * (i * a.heads + qh + head)) = make_float2(ref, inv);
                }
            }
        }
        if (a.scores && a.whole && a.hb == 1) {
            // The job's scores are this block's: its weights need no further launch.
            consumers_sync<THREADS>();
            whole_weights(kv, a, stats, scores, i, h, rows, s1, 32 * sub + lane, 32 * of_head);
        }
        if (tid == 0 && jobs.b0 == 0) {
            if (!whole) cut_job(a, jobs, i, end, total, per_seq);
            else if (a.by_job) a.split[3 * (i * per_seq + jobs.r)] = -1;
        }
        consumers_sync<THREADS>();   // buffers and queries are free again
    }
}

template <int DP, int NT>
struct Instance4 {
    // Units, heads and buffers are those of the other one too.  Blocks an SM are not: where lanes copy heads of 64 there
    // are two, and the rule of heads a unit for whole jobs counts three.
    using S = Shape<Packed<true>, DP, NT>;
    static AttendShape shape() { return {S::kHeads, DP, S::kUnit, S::kQHeads, S::kSlots, S::kBlocks}; }
    template <bool TMA>
    static mosaic_status go(const KvView &kv, AttendArgs a, const CUtensorMap &mk, const CUtensorMap &mv, int &blocks, cudaStream_t st) {
        using S = Shape<Packed<TMA>, DP, NT>;
        const int wave = resident<S, attend4_kernel<DP, NT, TMA>>();
        if (wave <= 0) return MOSAIC_ERR_CUDA;
        if (!a.whole && a.blocks > wave) a.blocks = wave;
        blocks = a.blocks;
        {
            KernelSpan span("attend4", st);
            const dim3 grid((unsigned)a.blocks), block(32 * (S::kWarps + S::kProducers));
            // More than one wave (whole jobs) must not stack up early.
            if (a.blocks <= wave) pdl_launch(attend4_kernel<DP, NT, TMA>, grid, block, S::kBytes, st, kv, a, mk, mv);
            else attend4_kernel<DP, NT, TMA><<<grid, block, S::kBytes, st>>>(kv, a, mk, mv);
        }
        return launch_status();
    }
    static mosaic_status launch(const mosaic_kv_cache &c, AttendArgs a, int &blocks, cudaStream_t st) {
        const KvView kv(c);
        alignas(64) CUtensorMap mk = {}, mv = {};
        a.out_quads = aligned16(a.out) && a.ldo % 4 == 0, a.q_quads = aligned16(a.q) && a.ldq % 4 == 0;
        // Positions are read 8 at a time.
        if (c.page_size % 8 == 0 && (!a.first || aligned16(c.position))) {
            auto maps = [&](int slots, int heads) {
                return pool_map<Q4>(&mk, c, c.k, slots, heads, &a.token_major, S::kRow) &&
                       pool_map<Q4>(&mv, c, c.v, slots, heads, &a.token_major, S::kRow);
            };
            a.box = 0;   // 16 slots of every head of a unit
            if (a.hpu > 1 && c.page_size % 16 == 0 && maps(16, a.hpu)) return go<true>(kv, a, mk, mv, blocks, st);
            // As many slots of a head as divide a page, 8 at least.
            for (a.box = a.hpu > 1 ? 16 : 64; c.page_size % a.box; a.box /= 2) {
            }
            if (maps(a.box, 1)) return go<true>(kv, a, mk, mv, blocks, st);
        }
        return go<false>(kv, a, mk, mv, blocks, st);
    }
};

// As with_instance.
template <class F>
auto with_instance4(int head_dim, int group, F f) {
    if (group <= 8) {
        if (head_dim <= 64) return f(Instance4<64, 1>());
        if (head_dim <= 128) return f(Instance4<128, 1>());
        return f(Instance4<256, 1>());
    }
    if (head_dim <= 64) return f(Instance4<64, 2>());
    if (head_dim <= 128) return f(Instance4<128, 2>());
    return f(Instance4<256, 2>());
}

}  // namespace

MOSAIC_ATTEND_TYPE(Q4, with_instance4)

}  // namespace mosaic
