// Attention of one new token per sequence over the paged cache: its
// mathematics and its split.  kv_attention_impl.cuh holds the kernel that reads
// the cache, kv_attention_<type>.cu its instances for an element type,
// kv_attention.cu the entry point and what follows the kernel.
//
//   s_j = scale q . k_j,  p = softmax(s) over the live slots,  out = sum p_j v_j
//
// Bound by reading K and V once (8 query heads a key/value head: 8 operations
// a byte of a 16-bit cache); the rest has to keep out of the copies' way.
//
//  * Two producer warps a block (four where lanes copy 4-bit rows) look pages up and fill a ring of units (16
//    rows a consumer warp, K and V) by tensor copies where rows share pages (a
//    lane issues one in about 100 cycles, so a box is as large as a page
//    allows: 64 x 16384 slots in pages of 16 took 436 us with one producer, 385
//    with two in a loop, 360 in straight code), else by 16-byte copies.  Consumer
//    warps only wait and multiply (a tile of 16 slots in about 800 cycles; with
//    its own copies a warp took 1600).
//  * S^T = K Q^T and O^T += V^T P^T on mma.sync with 8 query heads as the
//    narrow side: K and V fill the 16 rows whatever the group's size.  At 8
//    operations a byte the tensor pipe is a quarter busy, and registers are
//    where the softmax wants S, so tcgen05 would gain nothing here.
//  * fp32 queries and probabilities against 16-bit K and V: each is split
//    into terms of the cache's type (bf16: three terms, all 24 bits; fp16:
//    two, 22 bits), the products of which are exact; fp32 K and V into two tf32
//    terms (products of 22 bits).  fp16 terms are scaled by powers of two, the
//    lower one apart, and a tile with probabilities below 2^-29 takes those in
//    passes of their own (two unscaled terms of p 2^12 ended at 2^-37; now 16
//    heads of 128 a key/value head 70 -> 78 us on 32 x 4096, 8 heads 74 -> 75).  Terms are summed
//    from the least on in chains of at most six, and each chain's result is
//    added in fp32 with rounding to nearest, since the tensor cores truncate:
//    2e-7 to 5e-7 off the 64-bit result, as plain fp32 is 1e-7 to 1e-6.
//  * Softmax with a running maximum and sum a warp.  A unit holds slots of one,
//    two or four heads (hpu): with four a warp has a head to itself and no
//    warps are merged; with one they are, through shared memory.
//  * Work is cut evenly: the units of all (sequence, heads) jobs in a row, plus
//    a constant a job, in a contiguous share for every block of one wave.  A job
//    that lies in one block is finished there; one cut by a block's end leaves
//    partial sums that the join adds (at most two a block).  Short caches take
//    a block a job instead and need no join.
//
// Measured (device time, one GB300, copy rate 6.78 TB/s): 131071 slots of 8
// heads of 128 in bf16 6.3 TB/s in the kernel, 5.8 with launch and join; 64
// sequences of up to 16384 6.1; 48 of up to 2000 on 32 heads in fp16 6.0; fp32 8 x 6001
// 4.4, 32 x 6001 6.2; 37 slots 5.3 us.
#pragma once

#include "kv_cache.cuh"

namespace mosaic {

// Blocks of one wave at most (the resident ones of an instance are fewer).
constexpr int kAttendWave = 152 * 3;

struct AttendArgs {
    const float *q;
    int64_t ldq;
    const int32_t *lens, *first;
    int64_t max_len;
    int heads, group, hb;       // hb: blocks of query heads of a key/value head
    int hpu;                    // key/value heads of a unit (and of a job)
    int whole;                  // a block a job, nothing is cut
    int blocks;
    int job_cost;
    int token_major, box;       // of the tensor maps: heads lie closer than slots; slots of a box (0: a unit)
    float scale2, decay;        // scale * log2(e): scores are kept in the base-2 domain
    float *out;
    int64_t ldo;
    int q_quads, out_quads;     // rows of q and out are aligned words of four (4-bit caches)
    // Partial sums of a block: slot 2c (its first job, begun elsewhere) and
    // 2c + 1 (its last, ended elsewhere): maxima and sums, and outputs.
    float *part_ml, *part_o;
    int64_t *split;             // of block c: the job cut by its end (or -1), the last block with a part of
                                // it, and the units of the whole call
    int by_job;                 // split is of job j instead: the block whose end cuts it (or -1), and so on
    float *stats;               // final maximum and 1 / sum of (sequence, head), for the weights
    float *scores;              // (sequence, head) x score_rows, for the weights (none where 16 slots in a
                                // row do not count)
    int64_t score_rows;
    int quads;                  // four slots from a multiple of 4 on share a page and an aligned word of weights
};

// What the instance for a head_dim and a group has (query heads of a job,
// padded head_dim = row length of part_o, rows of a unit, key/value heads that
// a unit may hold: divisors of `most_heads` up to `buffers`, or all; blocks an
// SM); its launch on
// a.blocks blocks or one wave (`blocks`: how many); and whether a bounded wait
// of it ran out since the last call (after a stream sync).
struct AttendShape {
    int heads, dim, unit, most_heads, buffers, resident;
};
template <class T> AttendShape attend_shape(int head_dim, int group);
template <class T>
mosaic_status attend_launch(const mosaic_kv_cache &c, const AttendArgs &a, int &blocks, cudaStream_t st);
template <class T> mosaic_status attend_status();

namespace {

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }
// x, and NaN where x is infinite.
__device__ __forceinline__ float finite_or_nan(float x) {
    return fabsf(x) < __int_as_float(0x7f800000) ? x : __int_as_float(0x7fffffff);
}
// 2^x to 2^-22 relative; results below 2^-126 are zeros.
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace
}  // namespace mosaic
