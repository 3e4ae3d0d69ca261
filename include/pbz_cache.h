/*
 * pbz_cache -- a paged cache of keys and values held as compressed arrays, and attention taken on the compressed form.
 * Part of the pbz C ABI (pbz.h, whose conventions hold here: device pointers, caller's memory and stream, host checks
 * before any launch, status codes).
 *
 * A line is the D values of one head of one token, a block of a codec whose block shape is (D).  By orthonormality
 * (Sec. IV-A, Algorithm 6) a dot product of two lines is one of their coefficients, and a weighted sum of lines is the
 * inverse transform of the same sum of coefficients, so attention needs no decompressed key or value: the query is
 * transformed once, the result is transformed back once.
 *
 * The codec of a cache: one dimension, block extent D of 32, 64, 128 or 256 (PBZ_ERR_BLOCK_SHAPE otherwise), int8
 * indices, working type FP32, FP16 or bfloat16 (PBZ_ERR_TYPE), nothing pruned (PBZ_ERR_MASK); either transform.
 *
 * A pool of n_pages pages of page_size tokens (a power of two from 16 to 1024), for keys and for values:
 *   N  [n_pages][heads][page_size]       one working-type float a line
 *   F  [n_pages][heads][page_size][D]    int8
 * so a pool is the compressed form of a one-dimensional array, as pbz_compress writes it, and pbz_decompress reads it.
 * A sequence owns pages in the order of its table; its position j is at place j % page_size of page table[j / page_size],
 * and a slot is page * page_size + place.
 */
#ifndef PBZ_CACHE_H
#define PBZ_CACHE_H

#include "pbz.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pbz_cache {
  int64_t n_pages;
  int32_t heads;               /* heads of keys and values, 1 .. 65535 */
  int32_t page_size;
  void* k_N;                   /* device, 16-byte aligned, as are the others (PBZ_ERR_ALIGNMENT) */
  void* k_F;
  void* v_N;
  void* v_F;
} pbz_cache;

/* Bytes of one N and of one F pool.  Host only; the pointers in `cache` are not looked at. */
int pbz_cache_layout(const pbz_codec* codec, const pbz_cache* cache, size_t* n_bytes, size_t* f_bytes);

/* Compress n_tokens tokens' keys and values into their slots: per line C = x H, N = max |C|, F = rint(127 C / N).
 * Transform and binning are in FP64 whatever x's type, so that rounding borders fall as the definition has them; N is
 * rounded once, to the working type.  A line with a NaN or an infinity in it gives N = NaN, F = 0.
 *   k, v      device, element (t, h, d) at t * token_stride + h * head_stride + d; strides in elements, >= 0.  Any
 *             alignment of the element type; loads are wide where base and strides are multiples of 16 bytes.
 *   slots     device, n_tokens; a slot outside the pool (-1, say) leaves its token out.  Two tokens with one slot race.
 * More lines than a launch of 2^24 - 1 workgroups of 4096 / D takes are refused (PBZ_ERR_SHAPE), and likewise rows of q. */
typedef struct pbz_lines {
  const void* data;
  int64_t token_stride;
  int64_t head_stride;
} pbz_lines;
int pbz_cache_append(const pbz_codec* codec, const pbz_cache* cache, int64_t n_tokens, const pbz_lines* k,
                     const pbz_lines* v, pbz_ftype type, const int64_t* slots, void* stream);

/* Copy whole pages, keys and values: page pairs[2 i + 1] becomes what page pairs[2 i] is.
 *   pairs     host, read during the call.  Every page inside the pool, no page written twice, none written that is also
 *             read (PBZ_ERR_PAGES), so the order of the copies does not matter. */
int pbz_cache_copy_pages(const pbz_codec* codec, const pbz_cache* cache, int64_t n_pairs, const int32_t* pairs,
                         void* stream);

/* Attention of new tokens over the cache, their own keys and values among it (append them first):
 *   out_i = sum_j p_ij v_j,  p_ij = softmax over j of scale <q_i, k_j>,  k_j and v_j the decompressed lines.
 * Sequence b has its new tokens at rows starts[b] .. starts[b + 1) of q and out and lengths[b] cached positions; the new
 * tokens are its last ones.  Token i at position p sees j <= p (causal), and j > p - window (window > 0), among
 * 0 <= j < lengths[b]; a row that sees nothing is zero, its lse -infinity.  Rows of no sequence are zero, too.
 * Query head g reads the cache's head g / (q_heads / heads).
 * What is outside its bounds is not read: table entries outside the pool hide their positions, lengths beyond the table
 * are cut to it, starts to n_tokens.  Hidden positions' contents, whatever they are, do not reach the result (but for the
 * order of FP32 roundings: what weights refer to is renewed for several rows at a time); a line with an N that is not
 * finite makes the rows that see it not finite, and so may a key with an N of 2^97 or more (2^30 times N is a FP32 number
 * on the way).
 * Arithmetic: a query row is transformed in FP32 and held in 16-bit fixed point relative to its largest coefficient;
 * products with F are exact in integers; scores, running maxima and sums, and the output's sums are FP32 (scores have to be
 * within +-2^22, beyond which FP32 does not tell neighbours apart, and a row may come out not finite); a weight
 * (times N) is rounded to FP16 once, or held in two FP16 parts where q and out are FP16.  The unit of that is a power of
 * two, such that a row's largest weight times N is between 1 and 2^15 (above 2^-71, where another row's N is 2^32 or
 * more): what is smaller than 2^-14 of the former is off by 2^-25 of it. */
typedef struct pbz_attention {
  const void* q;               /* device, element (t, g, d) at t * q_token_stride + g * q_head_stride + d */
  void* out;                   /* device, likewise; must not overlap q */
  float* lse;                  /* device, [n_tokens][q_heads], natural logarithm of the sum of exponentials; may be NULL */
  pbz_ftype type;              /* of q and out: PBZ_BF16 or PBZ_F16 */
  int32_t q_heads;             /* a multiple of the cache's heads */
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
  int64_t n_tokens;            /* rows of q and out */
  int64_t n_seqs;
  const int32_t* starts;       /* device, n_seqs + 1, ascending; NULL: one token a sequence (n_tokens = n_seqs) */
  const int32_t* lengths;      /* device, n_seqs */
  const int32_t* table;        /* device, row b at b * table_stride */
  int64_t table_stride;        /* >= max_pages */
  int64_t max_pages;           /* columns of the table, at most 2^31 - 1024 positions */
  int64_t max_new;             /* what the longest run of new tokens is expected to be; work is dealt out by it */
  int64_t max_length;          /* likewise of lengths; 0: max_pages * page_size */
  int32_t causal;
  int64_t window;              /* 0: none */
  float scale;
} pbz_attention;
/* Bytes of workspace that the call takes.  Host only. */
int pbz_cache_attend_workspace(const pbz_codec* codec, const pbz_cache* cache, const pbz_attention* args, size_t* bytes);
/*   workspace   device, 16-byte aligned; contents on entry do not matter; not shared by calls that overlap. */
int pbz_cache_attend(const pbz_codec* codec, const pbz_cache* cache, const pbz_attention* args, void* workspace,
                     size_t workspace_bytes, void* stream);

/* Which sequence owns which page: host-side bookkeeping, no device work.  A page belongs to as many sequences as share
 * it after a fork, and is free when the last of them lets it go.  Calls on one handle may come from several threads. */
typedef struct pbz_pages pbz_pages;
int pbz_pages_create(pbz_pages** out, int64_t n_pages, int32_t page_size);
void pbz_pages_destroy(pbz_pages* pages);
int pbz_pages_open(pbz_pages* pages, int64_t* sequence);                       /* an empty sequence */
int pbz_pages_fork(pbz_pages* pages, int64_t sequence, int64_t* child);        /* shares every page */
int pbz_pages_close(pbz_pages* pages, int64_t sequence);                       /* PBZ_ERR_SEQUENCE when there is none */
/* Room for `tokens` more positions; slots (host, `tokens`) receives theirs.  Where the last page is partly filled and
 * shared, the sequence gets a page of its own: *n_copies is 1 and copy holds {from, to} for pbz_cache_copy_pages, to be
 * enqueued before the new tokens are appended; otherwise 0.  PBZ_ERR_PAGES, nothing changed, where pages are too few. */
int pbz_pages_extend(pbz_pages* pages, int64_t sequence, int64_t tokens, int64_t* slots, int32_t copy[2],
                     int32_t* n_copies);
/* Cut a sequence to its first `length` positions (PBZ_ERR_SHAPE when it has fewer). */
int pbz_pages_truncate(pbz_pages* pages, int64_t sequence, int64_t length);
int pbz_pages_length(const pbz_pages* pages, int64_t sequence, int64_t* length, int64_t* n_pages);
/* The sequence's pages in order; capacity entries of table are there, the ones past its pages are set to -1. */
int pbz_pages_table(const pbz_pages* pages, int64_t sequence, int32_t* table, int64_t capacity);
int pbz_pages_free_count(const pbz_pages* pages, int64_t* n_free);
/* Bring the pages in use to the front of the pool.  pairs (host, 2 * capacity) receives the {from, to} moves, *n_pairs
 * how many; every table changes with the call, so enqueue the copies before any later use.  At most as many moves as
 * half the pool's pages; PBZ_ERR_CAPACITY, nothing changed, when there are more than capacity. */
int pbz_pages_compact(pbz_pages* pages, int32_t* pairs, int64_t capacity, int64_t* n_pairs);

#ifdef __cplusplus
}
#endif
#endif /* PBZ_CACHE_H */
