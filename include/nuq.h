/*
 * nuq.h -- C ABI of the NUQSGD gradient-compression hot path for AMD MI355X (gfx950).
 *
 * The path (arXiv 1908.06077): per-bucket Euclidean norms -> nonuniform stochastic
 * quantization of |v_i|/||v|| onto the levels (0, 2^-s, ..., 1/2, 1) with sign
 * (Sec. 3.1, Def. 1) -> ENCODE into Elias-recursive-coded bit strings (App. A,
 * Alg. 2) -> DECODE, dequantize and average K workers' gradients (App. A; the
 * aggregate line of Alg. 1).  Beside it, the operators that training a transformer
 * on such gradients needs: AdamW, the gradients' norm, layer norm, dropout, the norms
 * around a block's residual sum, the loss over a vocabulary (near the end).
 *
 * Conventions for every entry point
 *   - Every data pointer is a DEVICE pointer owned by the caller, unless the
 *     comment says "host".  The library never frees or keeps them.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Calls enqueue work and
 *     return without synchronising, except nuq_last_error_flags.
 *   - Return value: NUQ_OK or a negative NUQ_E* code.  Argument errors are detected
 *     on the host before anything is enqueued.  Conditions only visible on the device
 *     (capacity overflow, non-finite norm, malformed stream) set sticky device flags
 *     read back with nuq_last_error_flags.
 *   - d = number of coordinates (>= 1), bucket = bucket size n (1..NUQ_MAX_BUCKET),
 *     B = ceil(d / bucket) buckets, bucket b covers [b*n, min((b+1)*n, d)),
 *     s = number of internal levels (1..NUQ_MAX_S), level index j in 0..s+1 with
 *     l_0 = 0 and l_j = 2^(j-1-s).
 *
 * Message layout produced by nuq_encode / nuq_quantize_encode (one per worker):
 *   norms[B]      fp32 bucket norms (the 32-bit ||v|| of App. A, kept beside the bits).
 *   bit_off[B+1]  u64.  bit_off[0] = 0.  Bucket b's records are stream bits
 *                 [start_b, bit_off[b+1]) with start_b = bit_off[b] rounded up to a
 *                 multiple of 32.
 *   words[W]      u32, W = ceil(bit_off[B] / 32).  Stream bit t is bit 31-(t%32) of
 *                 words[t/32].  Pad bits are zero.
 *   sync[B*nsync] u32 decoder index (this library's addition to the paper's message; the bit
 *                 strings do not depend on it), nsync = nuq_num_sync(bucket, sync_stride).  A bucket
 *                 is cut into blocks of NUQ_SYNC_BLOCK = 2048 coordinates and the records of every
 *                 block into P pieces of equal record count, P = the smallest power of two that is
 *                 at least min(bucket, 2048) / sync_stride (sync_stride = mean coordinates per
 *                 piece); nsync = ceil(bucket / 2048) * P.  With the bucket's records numbered in
 *                 index order, block t holding n_t of them from record f_t on, entry (t, g),
 *                 g = 0..P-1, stored at sync[b*nsync + t*P + g], describes record
 *                 f_t + floor(g * n_t / P): bits 0..20 = its bit offset from start_b (the bucket's
 *                 bit length if the bucket has no such record), bits 21..31 = its in-bucket index
 *                 minus 2048 t (0 if n_t = 0).  Piece (t, g) = the records from its entry's up to
 *                 the next entry's (or the bucket's end): a decoder parses every piece on its own,
 *                 taking the first record's index from the entry instead of from its gap code.
 *   A record, for a nonzero at in-bucket index i whose previous nonzero is at i_prev
 *   (-1 if none): ERC(i - i_prev), one sign bit (1 = negative), ERC(j).
 */
#ifndef NUQ_H
#define NUQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void *nuq_stream_t; /* hipStream_t */

enum {
    NUQ_OK = 0,
    NUQ_EINVAL = -1,     /* bad argument (size, range, NULL, misaligned)            */
    NUQ_ECAPACITY = -2,  /* a caller-provided buffer is too small (host-detectable) */
    NUQ_ENONFINITE = -3, /* reserved for host-side checks                           */
    NUQ_EHIP = -4        /* a HIP runtime call failed                               */
};

/* Sticky device flags (nuq_last_error_flags). */
enum {
    NUQ_FLAG_CAPACITY = 1,  /* encoded words did not fit words_cap; words is incomplete */
    NUQ_FLAG_NONFINITE = 2, /* a bucket norm was Inf/NaN; that bucket was encoded empty. A gradient norm or
                               new state of AdamW was: the step left that part as it was */
    NUQ_FLAG_MALFORMED = 4  /* a decoded stream broke the format, or nuq_encode refused a bucket; output is
                               incomplete.  Or a target of nuq_linear_cross_entropy_* lay outside the vocabulary */
};

/* A bucket's coordinates stay in the registers of one workgroup between the norm and the quantizer, so
 * that v is read from memory once: the largest workgroup (1024 threads) x 8 float4 = 32768 coordinates.
 * (The paper's bucket sizes are 8192 and 16384: Sec. 5, App. K.) */
#define NUQ_MAX_BUCKET 32768u
#define NUQ_MAX_S 14u
#define NUQ_MAX_WORKERS 32u /* K per nuq_decode_accumulate call */
#define NUQ_SYNC_BLOCK 2048u /* coordinates per block of the decoder index */

/* ---- sizes (pure host arithmetic, no device work) -------------------------------- */

/* B = ceil(d / bucket); 0 if bucket == 0. */
uint64_t nuq_num_buckets(uint64_t d, uint32_t bucket);

/* Decoder index entries per bucket of an ERC message: 0 if sync_stride == 0 (or not a power of two in
 * 64..1024), else ceil(bucket / 2048) * P with P as above. */
uint32_t nuq_num_sync(uint32_t bucket, uint32_t sync_stride);

/* The same for a Huffman-coded message (an entry per multiple of sync_stride inside the bucket):
 * 0 if sync_stride == 0, else ceil(bucket / sync_stride) - 1. */
uint32_t nuq_huffman_num_sync(uint32_t bucket, uint32_t sync_stride);

/* Upper bound on W for any input: every coordinate nonzero at the longest level code,
 * i.e. d * (2 + |ERC(s+1)|) bits, plus one word of padding per bucket. */
uint64_t nuq_max_words(uint64_t d, uint32_t bucket, uint32_t s);

/* Bytes of scratch the encoders need for K workers of these sizes (K = 1 for nuq_encode and
 * nuq_quantize_encode); 0 on invalid sizes. */
uint64_t nuq_encode_workspace_bytes(uint32_t K, uint64_t d, uint32_t bucket, uint32_t s);

/* Bytes of scratch that suffice for every entry point of this header at these sizes, whatever s:
 * nuq_encode_workspace_bytes(K, d, bucket, NUQ_MAX_S) (the decoders need none); 0 on invalid sizes. */
uint64_t nuq_workspace_bytes(uint64_t d, uint32_t bucket, uint32_t K);

/* ---- step 1: bucket norms (Def. 1: r_i = |v_i| / ||v||) --------------------------- */

/* norms[b] = sqrt(sum of v_i^2 over bucket b), rounded to fp32.
 * v: d floats, 4-byte aligned.  norms: B floats. */
int nuq_bucket_norms(const float *v, uint64_t d, uint32_t bucket, float *norms,
                     nuq_stream_t stream);

/* ---- step 2: quantizer (Def. 1; App. B eqs. h_case1, h_case2) --------------------- */

/* q[i] = level index j (bits 0..6) | sign (bit 7, 1 = negative, only if j > 0).
 * With r = |v_i| / norms[b] in bin [l_j, l_{j+1}) the result is j+1 with probability
 * p = (r - l_j) / (l_{j+1} - l_j), else j; the draw is the counter hash of
 * (seed, b, index in bucket) (24 uniform bits, "up" iff u / 2^24 < p, evaluated
 * exactly).  r >= 1 gives s+1; a zero norm or coordinate gives 0.
 * norms: B floats, normally the output of nuq_bucket_norms.  q: d bytes. */
int nuq_quantize(const float *v, uint64_t d, uint32_t bucket, uint32_t s, uint64_t seed,
                 const float *norms, uint8_t *q, nuq_stream_t stream);

/* ---- step 3: ENCODE (App. A; Alg. 2) ------------------------------------------------ */

/* Encodes the level/sign bytes q[d] into bit_off[B+1], words[<= words_cap] and, when
 * sync_stride != 0, sync[B*nsync] (sync may be NULL when sync_stride == 0).
 * sync_stride: 0, or a power of two in 64..1024.
 * workspace: at least nuq_encode_workspace_bytes(1, d, bucket, s) bytes, 16-byte aligned;
 * contents are scratch.  If the encoded size exceeds words_cap the device flag
 * NUQ_FLAG_CAPACITY is raised, bit_off is still complete and words holds the buckets
 * that fit.  A level index above s+1 in q is a caller error: it is coded modulo 16 (a multiple of 16 as
 * 1).  A bucket whose string such levels make longer than levels up to s+1 can (by more than the words its
 * place in the workspace is rounded up by) is refused: it becomes one word of ones, which no decoder takes,
 * its index entries are 0, NUQ_FLAG_MALFORMED is raised, and no other bucket changes. */
int nuq_encode(const uint8_t *q, uint64_t d, uint32_t bucket, uint32_t s, uint32_t sync_stride,
               uint64_t *bit_off, uint32_t *words, uint64_t words_cap, uint32_t *sync,
               void *workspace, uint64_t workspace_bytes, nuq_stream_t stream);

/* Steps 1-3 fused: v is read from memory once.  Outputs norms[B] as nuq_bucket_norms
 * would, and bit_off / words / sync exactly as nuq_encode(nuq_quantize(v, norms)) would.
 * A bucket whose norm is not finite is encoded as empty and raises NUQ_FLAG_NONFINITE. */
int nuq_quantize_encode(const float *v, uint64_t d, uint32_t bucket, uint32_t s, uint64_t seed,
                        uint32_t sync_stride, float *norms, uint64_t *bit_off, uint32_t *words,
                        uint64_t words_cap, uint32_t *sync, void *workspace,
                        uint64_t workspace_bytes, nuq_stream_t stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid it): nuq_quantize_encode with the workspace in a device array that is part of
 * the library itself, NUQ_STATIC_WORKSPACE_BYTES per GPU, held from the library's load to the end of
 * the process.  Same arguments otherwise, same kernels, same outputs bit for bit.  The call allocates
 * and frees nothing; its first call on a device looks the array's address up (make that call outside a
 * capture).  Sizes with nuq_encode_workspace_bytes(1, d, bucket, s) > NUQ_STATIC_WORKSPACE_BYTES are
 * rejected with NUQ_ECAPACITY before anything is enqueued (bucket 8192, s <= 5: up to 33.5 M
 * coordinates).  All calls on one GPU share the one array: calls that overlap in time (different
 * streams, or threads) race; calls on one stream do not.  Nothing in it has to be cleared between
 * calls: every word a call reads was written by that call. */
#define NUQ_STATIC_WORKSPACE_BYTES (32u << 20)
int nuq_quantize_encode_static(const float *v, uint64_t d, uint32_t bucket, uint32_t s, uint64_t seed,
                               uint32_t sync_stride, float *norms, uint64_t *bit_off, uint32_t *words,
                               uint64_t words_cap, uint32_t *sync, nuq_stream_t stream);

/* The same for K workers' gradients in one launch (the K simulated workers of Alg. 1 on one
 * device).  v, norms, bit_off, words, sync: HOST arrays of K device pointers; seeds, words_cap:
 * HOST arrays of K values.  Worker k's message equals what
 * nuq_quantize_encode(v[k], ..., seeds[k], ...) produces.  1 <= K <= NUQ_MAX_WORKERS.
 * workspace: at least nuq_encode_workspace_bytes(K, d, bucket, s) bytes. */
int nuq_quantize_encode_batch(uint32_t K, const float *const *v, const uint64_t *seeds, uint64_t d,
                              uint32_t bucket, uint32_t s, uint32_t sync_stride, float *const *norms,
                              uint64_t *const *bit_off, uint32_t *const *words,
                              const uint64_t *words_cap, uint32_t *const *sync, void *workspace,
                              uint64_t workspace_bytes, nuq_stream_t stream);

/* ---- step 4: DECODE + dequantize + aggregate (App. A DECODE; Alg. 1 aggregate) ------ */

/* out[i] = (accumulate ? out[i] : 0) + scale * sum_k norms_k[b] * sign * l_j, where
 * (sign, j) of coordinate i is decoded from worker k's bit string (0 if absent).
 * norms, bit_off, words, sync: HOST arrays of K device pointers (one message per
 * worker, all encoded with the same d, bucket, s, sync_stride); sync may be NULL or hold
 * NULLs when sync_stride == 0.  words_len: HOST array of K counts, the u32 words that
 * words[k] holds (as received).  1 <= K <= NUQ_MAX_WORKERS; average with scale = 1/K.
 * The sum over workers is taken in fp64 (in no fixed order, which cannot change it unless the
 * terms' exponents span more than 2^29), scaled in fp64 and rounded to fp32 once; with accumulate the
 * old out[i] is then added in fp32.  out: d floats.
 * A record that leaves its bucket's bit range or index range, a level index outside 1..s+1, or a
 * sync entry that contradicts the bit offsets raises NUQ_FLAG_MALFORMED and ends that part's
 * decoding.  So does a bucket whose offsets run backwards (bit_off[b+1] < bit_off[b]), end beyond
 * the words received (bit_off[b+1] > 32 * words_len[k]) or span 2^21 bits or more: such a bucket
 * contributes nothing and no word of it is read, so a cut-off or corrupted message cannot make the
 * kernels read outside words[k].  (norms, bit_off and sync are sized by d, bucket and sync_stride,
 * which the caller vouches for.) */
int nuq_decode_accumulate(uint32_t K, const float *const *norms, const uint64_t *const *bit_off,
                          const uint32_t *const *words, const uint64_t *words_len,
                          const uint32_t *const *sync, uint64_t d, uint32_t bucket, uint32_t s,
                          uint32_t sync_stride, float scale, int accumulate, float *out,
                          nuq_stream_t stream);

/* ---- other level sequences and the maximum norm (Sec. 3.1 before the special case; Sec. 4.1,
 *      "Generally spaced levels": exponential levels (0, p^s, ..., p, 1); uniform levels = QSGD,
 *      with the maximum norm = QSGDinf, Sec. 1 and Sec. 2) ------------------------------------ */

#define NUQ_NORM_L2 0u   /* Euclidean norm of the bucket */
#define NUQ_NORM_LINF 1u /* maximum norm of the bucket   */

/* A level table is s + 2 floats in HOST memory, 0 = levels[0] < levels[1] < ... < levels[s+1] = 1
 * (anything else: NUQ_EINVAL).  It is read during the call. */

/* norms[b] = max_i |v_i| over bucket b (exact; NaN if the bucket holds a NaN).  Arguments as
 * nuq_bucket_norms. */
int nuq_bucket_norms_linf(const float *v, uint64_t d, uint32_t bucket, float *norms,
                          nuq_stream_t stream);

/* nuq_quantize for the level sequence `levels`: with e_t = levels[t] * norms[b] and a = |v_i|,
 * j = largest t with e_t <= a (j = s+1: the top level), else j+1 iff
 * u * (e_{j+1} - e_j) < (a - e_j) * 2^24 over the real numbers (no rounding enters the decision), u the
 * 24-bit draw of nuq_quantize.  For levels[t] = 2^(t-1-s) q equals nuq_quantize's.  An infinite
 * coordinate takes the top level, a NaN level 0.
 * norms may come from nuq_bucket_norms or nuq_bucket_norms_linf; a zero or non-finite norm gives an
 * all-zero bucket.  q feeds nuq_encode unchanged (a level index is coded the same way whatever its
 * value). */
int nuq_quantize_table(const float *v, uint64_t d, uint32_t bucket, uint32_t s, const float *levels,
                       uint64_t seed, const float *norms, uint8_t *q, nuq_stream_t stream);

/* nuq_quantize_encode_batch for the level sequence `levels` and the norm `norm_kind` (NUQ_NORM_L2:
 * as nuq_bucket_norms; NUQ_NORM_LINF: as nuq_bucket_norms_linf): v is read once; worker k's norms are
 * what the norm entry point gives and its message is what
 * nuq_encode(nuq_quantize_table(v[k], ..., levels, seeds[k], norms[k])) gives.  Other arguments as
 * nuq_quantize_encode_batch. */
int nuq_quantize_encode_table_batch(uint32_t K, const float *const *v, const uint64_t *seeds, uint64_t d,
                                    uint32_t bucket, uint32_t s, const float *levels, uint32_t norm_kind,
                                    uint32_t sync_stride, float *const *norms, uint64_t *const *bit_off,
                                    uint32_t *const *words, const uint64_t *words_cap,
                                    uint32_t *const *sync, void *workspace, uint64_t workspace_bytes,
                                    nuq_stream_t stream);

/* nuq_decode_accumulate with l_j = levels[j]: out[i] = (accumulate ? out[i] : 0) +
 * scale * sum_k norms_k[b] * sign * levels[j].  Everything else as nuq_decode_accumulate. */
int nuq_decode_accumulate_table(uint32_t K, const float *const *norms, const uint64_t *const *bit_off,
                                const uint32_t *const *words, const uint64_t *words_len,
                                const uint32_t *const *sync, uint64_t d, uint32_t bucket, uint32_t s,
                                uint32_t sync_stride, const float *levels, float scale, int accumulate,
                                float *out, nuq_stream_t stream);

/* ---- fixed-width coding (Sec. 5: the "4-bit" and "8-bit" variants; 3 bits in Table 1) ------------ */

/* Every coordinate sends sign and level index in b bits, 3 <= b <= 8 with s + 2 <= 2^(b-1) (else
 * NUQ_EINVAL).  Message of one worker = norms[B] and packed[nuq_fixed_words(d, bucket, b)] u32:
 * coordinate i of a bucket is the code  sign << (b-1) | level index  at bits [i*b, i*b + b) of the
 * bucket's field, most significant bit first (bit t of a field = bit 31 - t%32 of its word t/32);
 * each bucket's field is ceil(bucket * b / 32) words (the short last bucket's too; unused bits 0). */
uint64_t nuq_fixed_words(uint64_t d, uint32_t bucket, uint32_t b);

/* packed <- the level|sign bytes q[d] (as nuq_quantize writes them). */
int nuq_pack_fixed(const uint8_t *q, uint64_t d, uint32_t bucket, uint32_t s, uint32_t b,
                   uint32_t *packed, nuq_stream_t stream);

/* Norms, quantizer and packing of K workers' gradients in one launch, v read once: norms[k] as
 * nuq_bucket_norms(v[k]) and packed[k] as nuq_pack_fixed(nuq_quantize(v[k], ..., seeds[k], norms[k])).
 * v, norms, packed: HOST arrays of K device pointers; seeds: HOST array.  1 <= K <= NUQ_MAX_WORKERS. */
int nuq_quantize_pack_fixed_batch(uint32_t K, const float *const *v, const uint64_t *seeds, uint64_t d,
                                  uint32_t bucket, uint32_t s, uint32_t b, float *const *norms,
                                  uint32_t *const *packed, nuq_stream_t stream);

/* out[i] = (accumulate ? out[i] : 0) + scale * sum_k norms_k[b] * sign * l_j from K fixed-width
 * messages (HOST arrays of K device pointers): fp64 sum in worker order, rounded to fp32 once.
 * A code with a level index above s+1, or a signed zero, raises NUQ_FLAG_MALFORMED. */
int nuq_unpack_accumulate_fixed(uint32_t K, const float *const *norms, const uint32_t *const *packed,
                                uint64_t d, uint32_t bucket, uint32_t s, uint32_t b, float scale,
                                int accumulate, float *out, nuq_stream_t stream);

/* The two fused calls above for a level sequence `levels` (s + 2 floats in HOST memory, as for
 * nuq_quantize_table) and the norm `norm_kind` (NUQ_NORM_L2 / NUQ_NORM_LINF): the fixed-width coding
 * of QSGD and QSGDinf (Sec. 1, Sec. 2; Sec. 5 compares the schemes at equal bit widths).  norms[k] is
 * what the norm entry point gives, packed[k] = nuq_pack_fixed(nuq_quantize_table(v[k], ..., levels,
 * seeds[k], norms[k])); the receiver sums norms_k[b] * sign * levels[j].  Other arguments, rounding
 * and flags as in the two calls above. */
int nuq_quantize_pack_fixed_table_batch(uint32_t K, const float *const *v, const uint64_t *seeds,
                                        uint64_t d, uint32_t bucket, uint32_t s, const float *levels,
                                        uint32_t norm_kind, uint32_t b, float *const *norms,
                                        uint32_t *const *packed, nuq_stream_t stream);
int nuq_unpack_accumulate_fixed_table(uint32_t K, const float *const *norms,
                                      const uint32_t *const *packed, uint64_t d, uint32_t bucket,
                                      uint32_t s, const float *levels, uint32_t b, float scale,
                                      int accumulate, float *out, nuq_stream_t stream);

/* ---- Huffman-coded levels (Sec. 5, "Efficient Encoding": a Huffman code for the level indices, built
 *      from a sample and then kept) ------------------------------------------------------------------ */

/* hist[0..15] (DEVICE, overwritten) <- how often each level index occurs in the level|sign bytes q[d]. */
int nuq_level_histogram(const uint8_t *q, uint64_t d, uint64_t *hist, nuq_stream_t stream);

/* Host arithmetic.  lengths[0..s+1] <- code lengths from the histogram hist[0..s+1] (both HOST):
 * Huffman's algorithm on hist[j] + 1 (a level the sample never showed still gets a code), merging
 * the two smallest nodes by (weight, id), a leaf's id being its symbol, the k-th merged node's id
 * s + 2 + k.  Lengths are 1..s+1.  The codewords are the canonical ones: symbols by (length, symbol),
 * the first is 0, each next one (previous + 1) shifted left by the increase in length. */
int nuq_huffman_lengths(const uint64_t *hist, uint32_t s, uint8_t *lengths);

/* Capacity that always suffices for nuq_encode_huffman's words, and its workspace size. */
uint64_t nuq_huffman_max_words(uint64_t d, uint32_t bucket);
uint64_t nuq_encode_huffman_workspace_bytes(uint64_t d, uint32_t bucket);

/* Message of the bytes q[d] under the code `lengths` (HOST, s + 2 values; NUQ_EINVAL unless they give a
 * complete prefix code): per bucket, for every coordinate in order, the codeword of its level index
 * (most significant bit first), then its sign bit when the level is not zero.  bit_off[B+1], words,
 * word alignment, capacity flag and workspace alignment as for nuq_encode.  sync[B * nsync],
 * nsync = nuq_huffman_num_sync(bucket, sync_stride): entry (b, g), g = 1..nsync, at sync[b*nsync + g-1]
 * = bit offset, from the bucket's start, of coordinate g * sync_stride (the bucket's bit length where
 * the bucket ends before it). */
int nuq_encode_huffman(const uint8_t *q, uint64_t d, uint32_t bucket, uint32_t s, uint32_t sync_stride,
                       const uint8_t *lengths, uint64_t *bit_off, uint32_t *words, uint64_t words_cap,
                       uint32_t *sync, void *workspace, uint64_t workspace_bytes, nuq_stream_t stream);

/* Norms, quantizer and Huffman coding of K workers' gradients in one launch, v read once: norms[k] as
 * nuq_bucket_norms(v[k]) and the message as nuq_encode_huffman(nuq_quantize(v[k], ..., seeds[k],
 * norms[k])).  Array arguments as nuq_quantize_encode_batch; workspace of at least
 * nuq_encode_huffman_batch_workspace_bytes(K, d, bucket, s) bytes, 16-byte aligned. */
uint64_t nuq_encode_huffman_batch_workspace_bytes(uint32_t K, uint64_t d, uint32_t bucket, uint32_t s);
int nuq_quantize_encode_huffman_batch(uint32_t K, const float *const *v, const uint64_t *seeds, uint64_t d,
                                      uint32_t bucket, uint32_t s, uint32_t sync_stride,
                                      const uint8_t *lengths, float *const *norms, uint64_t *const *bit_off,
                                      uint32_t *const *words, const uint64_t *words_cap,
                                      uint32_t *const *sync, void *workspace, uint64_t workspace_bytes,
                                      nuq_stream_t stream);

/* q[d] <- the level|sign bytes of such a message.  A segment that does not end where the next one
 * starts, a prefix that is no codeword, or a sync entry out of order raises NUQ_FLAG_MALFORMED. */
int nuq_decode_huffman(const uint64_t *bit_off, const uint32_t *words, const uint32_t *sync, uint64_t d,
                       uint32_t bucket, uint32_t s, uint32_t sync_stride, const uint8_t *lengths,
                       uint8_t *q, nuq_stream_t stream);

/* The same for K messages in one launch (bit_off, words, sync, q: HOST arrays of K device pointers;
 * one code for all).  1 <= K <= NUQ_MAX_WORKERS. */
int nuq_decode_huffman_batch(uint32_t K, const uint64_t *const *bit_off, const uint32_t *const *words,
                             const uint32_t *const *sync, uint64_t d, uint32_t bucket, uint32_t s,
                             uint32_t sync_stride, const uint8_t *lengths, uint8_t *const *q,
                             nuq_stream_t stream);

/* nuq_decode_accumulate for K Huffman-coded messages (Sec. 5, "Efficient Encoding"; App. A DECODE;
 * Alg. 1 aggregate) in one launch: out[i] = (accumulate ? out[i] : 0) + scale * sum_k norms_k[b] *
 * sign * 2^(j-1-s), (sign, j) decoded from worker k's string; the level|sign bytes are never written.
 * Arguments, summation, rounding and NUQ_FLAG_MALFORMED as nuq_decode_accumulate (words_len included),
 * lengths as nuq_encode_huffman.  Geometry: bucket > sync_stride (the messages carry an index), and
 * the pieces of the K messages of a 2048-coordinate tile must fit the tile's 64 parsing lanes with a
 * power-of-two group of lanes per message: for bucket > 2048, K' * 2048 / sync_stride <= 64 with K' =
 * K rounded up to a power of two (K <= 8 at stride 256); else NUQ_EINVAL, and the caller uses
 * nuq_decode_huffman_batch + nuq_average_levels. */
int nuq_decode_accumulate_huffman(uint32_t K, const float *const *norms, const uint64_t *const *bit_off,
                                  const uint32_t *const *words, const uint64_t *words_len,
                                  const uint32_t *const *sync, uint64_t d, uint32_t bucket, uint32_t s,
                                  uint32_t sync_stride, const uint8_t *lengths, float scale, int accumulate,
                                  float *out, nuq_stream_t stream);

/* out[i] = (accumulate ? out[i] : 0) + scale * sum_k norms_k[b] * sign * l_j from K arrays of
 * level|sign bytes (norms, q: HOST arrays of K device pointers): the aggregate of Alg. 1 for messages
 * already decoded to bytes.  fp64 sum in worker order, rounded to fp32 once. */
int nuq_average_levels(uint32_t K, const float *const *norms, const uint8_t *const *q, uint64_t d,
                       uint32_t bucket, uint32_t s, float scale, int accumulate, float *out,
                       nuq_stream_t stream);

/* ---- parameter update and variance diagnostic (Alg. 1 aggregate; Sec. 4.2; App. J) --------------- */

/* The plain aggregate step of Alg. 1 with Omega = R^d,  w <- w - (alpha/K) sum_k Q_k,  is
 * nuq_decode_accumulate (or its table / fixed-width / byte variants) with out = w, accumulate = 1 and
 * scale = -alpha/K: no separate pass over w.
 *
 * Momentum rule of Sec. 4.2 on d fp32 values in DEVICE memory, g the averaged gradient:
 *   y = w - alpha g;  y^l = w - l alpha g;  w <- y + mu (y^l - yl);  yl <- y^l.
 * l = 0 is heavy ball, l = 1 Nesterov's method.  The caller sets yl = w before the first step and owns
 * all three arrays; w and yl are updated in place.  Evaluated in fp64 in this order from the fp32
 * inputs, one rounding per stored value.  NUQ_EINVAL for a null pointer with d > 0, a non-finite
 * alpha, mu or l, or mu outside [0, 1). */
int nuq_momentum_step(float *w, float *yl, const float *g, uint64_t d, float alpha, float mu, float l,
                      nuq_stream_t stream);

/* nuq_decode_accumulate and nuq_momentum_step in one launch: (w, yl) <- momentum rule with
 * g[i] = the fp32 value nuq_decode_accumulate(..., scale, accumulate = 0, ...) would store at i (scale =
 * 1/K for Alg. 1's average).  Same bits in w and yl as the two calls give; the average itself is not
 * stored, which saves its write and read (8 of the update's 24 bytes per coordinate).  Message
 * arguments as nuq_decode_accumulate; alpha, mu, l, w, yl as nuq_momentum_step. */
int nuq_decode_momentum_step(uint32_t K, const float *const *norms, const uint64_t *const *bit_off,
                             const uint32_t *const *words, const uint64_t *words_len,
                             const uint32_t *const *sync, uint64_t d, uint32_t bucket, uint32_t s,
                             uint32_t sync_stride, float scale, float alpha, float mu, float l, float *w,
                             float *yl, nuq_stream_t stream);

/* First and second moments of a gradient estimate across draws (App. J): sum[i] += g[i],
 * sumsq[i] += g[i]^2 in fp64; g, sum, sumsq: DEVICE arrays of d values, sum and sumsq zeroed by the
 * caller before the first draw. */
int nuq_moments_accumulate(const float *g, double *sum, double *sumsq, uint64_t d, nuq_stream_t stream);

/* Mean normalized variance of App. J after M >= 1 draws: out2[0] = sum_i (sumsq_i/M - (sum_i/M)^2),
 * out2[1] = sum_i sumsq_i/M (DEVICE doubles); the diagnostic is out2[0] / out2[1] (the two means over
 * coordinates share the factor 1/d).  Variance = mean squared deviation from the mean of the M draws.
 * workspace: DEVICE memory of at least NUQ_VARIANCE_WORKSPACE_BYTES bytes, 8-byte aligned, overwritten.
 * The summation order is fixed: equal inputs give equal bits. */
#define NUQ_VARIANCE_WORKSPACE_BYTES 16384u
int nuq_normalized_variance(const double *sum, const double *sumsq, uint64_t d, uint64_t M, void *workspace,
                            uint64_t workspace_bytes, double *out2, nuq_stream_t stream);

/* ---- training of transformers: AdamW, the gradients' norm, layer norm ------------------------------ */

/* Element types. */
#define NUQ_F32 0u
#define NUQ_BF16 1u
#define NUQ_F16 2u

/* The norm of T tensors taken as one vector, and the factor that clips them.  g: HOST array of T device
 * pointers, element-aligned (NULL where n is 0); n: HOST array of T counts; type: NUQ_F32, NUQ_BF16 or
 * NUQ_F16.  out (DEVICE, 2 floats): out[0] = sqrt(sum of all g_i^2), out[1] = min(1, max_norm / out[0]).
 * Summed in fp64 in an order that depends on the sizes and on which tensors lie directly behind one another
 * in memory (those are taken as one): the same tensors give the same bits, equal values elsewhere the same
 * norm but for the rounding of fp64 sums, rounded once to fp32.  No square overflows.  Where the norm is not
 * finite (or above the largest float) out[1] is NaN, which the steps below take as "leave everything as it
 * is", and NUQ_FLAG_NONFINITE is raised.  max_norm: positive,
 * infinite for the norm alone (NUQ_EINVAL otherwise, also for more than 2^19 tensors none of which lies
 * behind another).  workspace: DEVICE memory of at least
 * NUQ_GRADIENT_NORM_WORKSPACE_BYTES bytes, 8-byte aligned, overwritten. */
#define NUQ_GRADIENT_NORM_WORKSPACE_BYTES 65536u
int nuq_gradient_norm(uint32_t T, const void *const *g, const uint64_t *n, uint32_t type, float max_norm,
                      void *workspace, uint64_t workspace_bytes, float *out, nuq_stream_t stream);

/* One AdamW step on T tensors at once; step t = 1, 2, ... of the tensors' states.  Per element, with
 * lambda = decay[i] of its tensor and c = *coefficient (1 without):
 *   g = c * gradient;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2;
 *   w <- w (1 - alpha lambda) - alpha / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps).
 * w, g, m, v: HOST arrays of T device pointers to n[i] elements each (element-aligned; NULL where n[i]
 * is 0), w, m, v fp32, g of type g_type; the arrays of a call must not overlap.  copy: NULL, or a HOST
 * array of T device pointers to n[i] elements of copy_type (NUQ_BF16 or NUQ_F16): the new w, rounded
 * to nearest, for a model that computes in 16 bits.  decay: HOST array of T, NULL for none.
 * coefficient: DEVICE float, or NULL: nuq_gradient_norm's out + 1, or a scale that gradients were
 * multiplied with, inverted.
 * Evaluated in fp32, one rounding per product and sum in m and v; w within a few units of the last
 * place of the subtracted term.  An element whose new m or v would not be finite keeps w, m and v
 * (its copy is still written) and raises NUQ_FLAG_NONFINITE.
 * NUQ_EINVAL: t = 0; beta outside [0, 1); eps below 2^-126; alpha, beta, decay, or what is made of them
 * in fp32, not finite. */
int nuq_adamw_step(uint32_t T, float *const *w, const void *const *g, float *const *m, float *const *v,
                   void *const *copy, const uint64_t *n, const float *decay, uint32_t g_type,
                   uint32_t copy_type, double alpha, double beta1, double beta2, double eps, uint64_t t,
                   const float *coefficient, nuq_stream_t stream);

/* The same with m and v held in 8 bits.  A tensor's elements are cut into blocks of NUQ_STATE_BLOCK (the
 * last one short); scales[i] holds 2 * nuq_state_blocks(n[i]) floats, for block b  a = scales[2b] = its
 * largest |m| and  e = scales[2b+1] = its largest v, both 0 where below 2^-126.  Code k of
 *   m (n[i] bytes, OCP float8 e4m3): stands for  e4m3(k) * (a * 2^-8); stored is a code for m * (1/a) * 256;
 *   v (n[i] bytes, unsigned float, 5 bits of exponent, 3 of fraction): stands for
 *     float(bits k << 20) * 2^96 * e; stored is a code k whose float(bits k << 20), which may be
 *     subnormal, is next to v * (1/e) * 2^-96, at least 1 where v > 0;
 * each product and quotient rounded to fp32.  A step replaces the share (1 - beta) / (1 - beta^t) of m, of v.
 * Where that is 1/16 or more, the code is the nearest, ties to even.  Where it is less (beta2 = 0.999 from
 * t = 17 on), the nearest code could be the old one for good, and the code is drawn instead: one of the two
 * next to the value, so that the mean is the value (to 2^-16 of a step); what is within 7 units of the last
 * place of a code's value gets that code.  Draws come from t, the block's new a and e and the element's place
 * in its block: equal inputs give equal bits.  The largest element of a block is held exactly.  With
 * gradients of one size and beta2 = 0.999, sqrt(v) is held to some 12 % (standard deviation), without bias.
 * All zeros (codes and scales) is the state before step 1.  The step uses the new m and
 * v before they are rounded to codes.  A block with a new m or v that is not finite keeps w, codes and
 * scales (its copy is still written) and raises NUQ_FLAG_NONFINITE.  Other arguments and errors as above. */
#define NUQ_STATE_BLOCK 256u
uint64_t nuq_state_blocks(uint64_t n);
int nuq_adamw_step_coded(uint32_t T, float *const *w, const void *const *g, uint8_t *const *m,
                         uint8_t *const *v, float *const *scales, void *const *copy, const uint64_t *n,
                         const float *decay, uint32_t g_type, uint32_t copy_type, double alpha,
                         double beta1, double beta2, double eps, uint64_t t, const float *coefficient,
                         nuq_stream_t stream);

/* m[n], v[n] (DEVICE floats) <- the values that the codes of one tensor stand for. */
int nuq_adamw_state_values(const uint8_t *m_codes, const uint8_t *v_codes, const float *scales, uint64_t n,
                           float *m, float *v, nuq_stream_t stream);

/* Layer norm of `rows` rows of `hidden` elements.  With s = x, or s = x + residual rounded to x's type
 * and stored in total:  mean, var of the row (divided by hidden);  rstd = 1 / sqrt(var + eps);
 * y = (s - mean) * rstd * weight + bias.
 * x, residual, total, y: DEVICE, of `type`, element-aligned, row r at r * ld elements (ldx, ldr: any;
 * ldt, ldy: at least hidden).  residual and total: both or neither.  weight, bias: hidden elements of
 * weight_type (`type` or NUQ_F32), each may be NULL.  mean, rstd: `rows` floats each, may be NULL.
 * y may be x, total may be x or residual, at the same stride.  rows below 2^31, hidden at most 2^30.  Statistics in fp32, the
 * variance from centred values.  eps: finite, not negative. */
int nuq_layer_norm_forward(const void *x, uint64_t ldx, const void *residual, uint64_t ldr,
                           const void *weight, const void *bias, uint64_t rows, uint32_t hidden, float eps,
                           uint32_t type, uint32_t weight_type, void *total, uint64_t ldt, void *y,
                           uint64_t ldy, float *mean, float *rstd, nuq_stream_t stream);

/* Its gradients, from dy, the forward's s (x, or total) and its mean and rstd.  With n = (s - mean) * rstd
 * and d = dy * weight:  dx = rstd * (d - mean(d) - n * mean(d n)) (+ add), the gradient of x and of
 * residual alike; add: the gradient that arrives through total, may be NULL.  dweight = sum over rows of
 * dy * n, dbias = sum of dy (hidden elements of weight_type, each may be NULL): summed in fp32 in a fixed
 * order, with at most rows / 256 + 64 roundings of the summed magnitudes, rounded once.  dx may be dy, at the same stride.  Row strides as above (ldg of dy, ldx, lda of add: any; ldd of dx
 * at least hidden).  workspace: DEVICE memory, nuq_layer_norm_workspace_bytes(rows, hidden) bytes,
 * 16-byte aligned, overwritten; may be NULL where neither dweight nor dbias is asked for. */
uint64_t nuq_layer_norm_workspace_bytes(uint64_t rows, uint32_t hidden);
int nuq_layer_norm_backward(const void *dy, uint64_t ldg, const void *x, uint64_t ldx, const void *weight,
                            const float *mean, const float *rstd, const void *add, uint64_t lda,
                            uint64_t rows, uint32_t hidden, uint32_t type, uint32_t weight_type, void *dx,
                            uint64_t ldd, void *dweight, void *dbias, void *workspace,
                            uint64_t workspace_bytes, nuq_stream_t stream);

/* ---- between the blocks of a transformer: dropout, norms around the residual sum -------------------- */

/* Dropout of `rows` rows of `hidden` elements, from a mask that is computed and never stored.  Element (r, c) is kept iff
 * u >= T, T = floor(p 2^24 + 1/2), u the upper 24 bits of a hash of (seed, *step, r, c): with
 *   z = seed + *step * 0xD1342543DE82EF95 + (r + 1) * 0x9E3779B97F4A7C15                       (modulo 2^64)
 *   z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9;  z = (z ^ z >> 27) * 0x94D049BB133111EB;  z ^= z >> 31
 *   x = ((uint32_t)z + c) * 0x9E3779B1;  x = (x ^ x >> 15 ^ z >> 32) * 0x85EBCA6B;  u = (x ^ x >> 16) >> 8      (modulo 2^32)
 * y = (kept ? x * 2^24 / (2^24 - T) : 0) + residual, in fp32, rounded once.  What is dropped counts as 0, also a NaN.  The gradient
 * is the same call on dy, without a residual: the same seed and step give the same mask.  p: 0 (all is kept) to 1.  step: DEVICE
 * int64, NULL for 0; it is read when the kernel runs, so that a captured graph draws anew where the program moves it.
 * x, residual (may be NULL), y: DEVICE, of `type`, element-aligned, row r at r * ld elements (ldx, ldr: any; ldy: at least hidden).
 * y may be x or residual, at the same stride (NUQ_EINVAL otherwise).  rows and hidden below 2^31. */
int nuq_dropout(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, uint64_t rows, uint32_t hidden,
                uint32_t type, double p, uint64_t seed, const int64_t *step, void *y, uint64_t ldy, nuq_stream_t stream);

/* The seam between two blocks: the norm of a branch x (inner), gate, dropout, scales and the residual sum, and the norm of the sum
 * (outer) that the next block begins with.  Per row
 *   n1 = N(x), b = n1 * inner_weight + inner_bias        (without an inner norm b = x)
 *   total = residual_scale * residual + scale * drop(gate * b), rounded to `type`
 *   y = N(total) * outer_weight + outer_bias             (without an outer norm there is no y)
 * N(s) = (s - mean) / sqrt(mean of (s - mean)^2 + eps); NUQ_RMS_NORM takes 0 for the mean.  drop: as nuq_dropout, of the same element
 * (r, c).  inner, outer: NUQ_NO_NORM, NUQ_LAYER_NORM or NUQ_RMS_NORM, one of them at least a norm.  residual may be NULL (taken as
 * 0), and so may each weight, bias and the gate: `hidden` elements of weight_type (`type` or NUQ_F32).  stats: [4][rows] floats, or
 * NULL: the inner norm's mean and 1 / sqrt(...), the outer norm's; what a norm does not have is not written.
 * Rows and strides as in nuq_layer_norm_forward; y may be x, total may be x or residual, at the same stride (NUQ_EINVAL otherwise).  rows
 * below 2^31, hidden at most NUQ_RESIDUAL_NORM_MAX_HIDDEN.  In fp32 throughout, variances from centred values, total and y rounded once;
 * eps: finite, not negative; scale, residual_scale: finite. */
#define NUQ_NO_NORM 0u
#define NUQ_LAYER_NORM 1u
#define NUQ_RMS_NORM 2u
#define NUQ_RESIDUAL_NORM_MAX_HIDDEN 16384u
int nuq_residual_norm_forward(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, uint32_t inner,
                              const void *inner_weight, const void *inner_bias, const void *gate, uint32_t outer,
                              const void *outer_weight, const void *outer_bias, uint64_t rows, uint32_t hidden,
                              float eps, float scale, float residual_scale, double p, uint64_t seed,
                              const int64_t *step, uint32_t type, uint32_t weight_type, void *total, uint64_t ldt,
                              void *y, uint64_t ldy, float *stats, nuq_stream_t stream);

/* Its gradients, from dy (NULL without an outer norm), dtotal, the gradient that arrives through total (may be NULL where there is
 * an outer norm), the forward's x, total and stats, and the same vectors, scales, p, seed and step.  With n2 = N(total), d = dy *
 * outer_weight, rstd the outer norm's:
 *   dt = dtotal + rstd * (d - mean(d) - n2 * mean(d n2));   dresidual = residual_scale * dt (may be NULL)
 *   g = scale * drop(dt);  h = g * gate;   dx = rstd1 * (h' - mean(h') - n1 * mean(h' n1)),  h' = h * inner_weight  (or h)
 * (mean(d) and mean(h') fall away with NUQ_RMS_NORM), and the sums over rows, each of which may be NULL:  dinner_weight of h n1,
 * dinner_bias of h, dgate of g b, douter_weight of dy n2, douter_bias of dy: in fp32 in a fixed order, with at most rows / 256 + 64
 * roundings of the summed magnitudes (of g n1 and g, times the vectors that are constant along the sum), rounded once.  dx may be dy or
 * x, dresidual may be dtotal or total, at the same stride, and not where a sum is asked for over more than 8192 columns (NUQ_EINVAL
 * otherwise); the two must not overlap.  workspace: DEVICE memory of nuq_residual_norm_workspace_bytes(rows, hidden) bytes, 16-byte aligned,
 * overwritten; may be NULL where no sum is asked for. */
uint64_t nuq_residual_norm_workspace_bytes(uint64_t rows, uint32_t hidden);
int nuq_residual_norm_backward(const void *dy, uint64_t ldg, const void *dtotal, uint64_t lda, const void *x, uint64_t ldx,
                               const void *total, uint64_t ldt, uint32_t inner, const void *inner_weight,
                               const void *inner_bias, const void *gate, uint32_t outer, const void *outer_weight,
                               uint64_t rows, uint32_t hidden, float scale, float residual_scale, double p, uint64_t seed,
                               const int64_t *step, uint32_t type, uint32_t weight_type, const float *stats, void *dx,
                               uint64_t ldd, void *dresidual, uint64_t lde, void *dinner_weight, void *dinner_bias,
                               void *dgate, void *douter_weight, void *douter_bias, void *workspace,
                               uint64_t workspace_bytes, nuq_stream_t stream);

/* ---- the loss of a language model ----------------------------------------------------------------- */

/* Softmax cross entropy of `rows` rows x of `hidden` elements against the `vocab` rows of weight, z = x weight^T, without z in memory.
 * With t = target[r], e = smoothing, per row
 *   lse = log sum over v of exp(z_v);   loss = lse - (1 - e) z_t - e mean(z)
 * and 0 for a row whose target is `ignore`.  A target outside the vocabulary that is not `ignore` makes the row's loss NaN and raises
 * NUQ_FLAG_MALFORMED.  x, weight: DEVICE, of `type`, element-aligned, row r at r * ld elements (ldx, ldw: any).  target: DEVICE int64.
 * loss (may be NULL), lse: `rows` floats.  mean (may be NULL): 2 floats, the mean loss over the rows that are not ignored, and 1 / their
 * number (0 and 1 where there are none).  Products of operands of 16 bits are exact and summed in fp32 on the matrix cores, fp32 operands
 * are multiplied in fp32; exponentials and sums in fp32, the mean in fp64 in a fixed order.  rows at most 2^20, hidden 2^16, vocab 2^24,
 * rows * vocab 2^38; smoothing from 0, below 1.  workspace: DEVICE memory of nuq_linear_cross_entropy_workspace_bytes(..., 0) bytes,
 * 16-byte aligned, overwritten; it holds two or three numbers per row and 64 to 256 entries of the vocabulary, and a copy of x or weight
 * where 16-byte loads do not take it as it stands (its address, stride or width no multiple of 16 bytes). */
uint64_t nuq_linear_cross_entropy_workspace_bytes(const void *x, uint64_t ldx, const void *weight, uint64_t ldw,
                                                  uint64_t rows, uint32_t hidden, uint32_t vocab, uint32_t type,
                                                  int backward);
int nuq_linear_cross_entropy_forward(const void *x, uint64_t ldx, const void *weight, uint64_t ldw, uint64_t rows,
                                     uint32_t hidden, uint32_t vocab, uint32_t type, const int64_t *target, int64_t ignore,
                                     float smoothing, float *loss, float *lse, float *mean, void *workspace,
                                     uint64_t workspace_bytes, nuq_stream_t stream);

/* Its gradients, from the forward's lse:  with g the gradient of a row's loss, 0 where the target is `ignore` or outside the vocabulary,
 *   d_v = exp(z_v - lse) - e / vocab - (1 - e) [v = t];   dx = g sum over v of d_v weight_v;   dweight_v = sum over rows of g d_v x
 * dx: rows at ldd >= hidden elements, dweight: vocab rows at lde >= hidden, of `type`, each may be NULL; they must not overlap the
 * inputs.  g = *grad, or grad[r] where grad_per_row, times mean[1] where there is a mean (the forward's: the gradient of the mean loss).
 * The logits are made again, a piece of the vocabulary at a time.  d is rounded to `type` (fp16: 2^14 d), sums are fp32, and results are
 * rounded once.  For dweight with grad_per_row x times g over the largest |g| of the rows that count is rounded to `type` too.  A row that
 * does not count takes no part, whatever x and grad hold there.  The order of all sums is fixed.  workspace: as above, of
 * nuq_linear_cross_entropy_workspace_bytes(..., 1) bytes: a copy of x, d of a piece of the vocabulary (at most 320 MiB, or 2048 entries
 * where these are more: 4 GiB at 2^20 rows of 16 bits, 8 GiB in fp32), and sums of dx in fp32, several where x is small. */
int nuq_linear_cross_entropy_backward(const void *x, uint64_t ldx, const void *weight, uint64_t ldw, uint64_t rows,
                                      uint32_t hidden, uint32_t vocab, uint32_t type, const int64_t *target,
                                      int64_t ignore, float smoothing, const float *lse, const float *grad,
                                      int grad_per_row, const float *mean, void *dx, uint64_t ldd, void *dweight,
                                      uint64_t lde, void *workspace, uint64_t workspace_bytes, nuq_stream_t stream);

/* ---- errors ---------------------------------------------------------------------- */

/* Waits for `stream`, copies the sticky device flags of the current device to
 * *host_flags (host pointer) and clears them. */
int nuq_last_error_flags(uint32_t *host_flags, nuq_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* NUQ_H */
