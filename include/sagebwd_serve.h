/*
 * sagebwd_serve.h -- C ABI of the operators around the attention of sagebwd.h that training and serving a model
 * need beside it, on one MI355X (gfx950): rotary positions, and a paged key/value cache held in 4 bits with its
 * bookkeeping and the attention that reads it.
 *
 * The conventions of sagebwd.h hold: device pointers of the caller, nothing allocated, no memset, no host
 * synchronisation, no state between calls; work is enqueued on `stream` and may be captured; arguments are checked on
 * the host before anything is launched and a sagebwd_status comes back.  What lies in device memory (lengths,
 * positions, page numbers) cannot be checked there: the kernels bound it, as each call says, so that wrong values
 * give wrong results and no access outside the tensors.  Tensors of one call do not overlap unless a call says so.
 *
 * The order of a step of serving:  sagebwd_cache_plan (lengths -> pages, slots, positions), sagebwd_rotary (Q, K),
 * sagebwd_cache_append (K, V -> cache), sagebwd_cache_attention (Q, cache -> O).  The four repeat themselves bit for bit.
 *
 * ---- the cache -----------------------------------------------------------------------------------------------
 * A pool of `pages` pages, bytes [pages, H, page * (d + 4 d / group)], 16-byte aligned.  A page holds `page` tokens of
 * each of the H key/value heads; a head's part holds K's codes (page * d / 2 bytes), V's codes (the same), K's scales
 * and V's scales (page * d / group * 2 bytes each).  A value is (nibble - 8) * scale.
 *   K's codes    token t, channel c = 32 j + 8 p + r: nibble r / 2 + 4 (r % 2) of the 32-bit word at byte
 *                t * d / 2 + p * d / 8 + 4 j
 *   V's codes    token t = 8 o + i, channel c = 64 h + 16 j + m: nibble j of the 16-bit word at byte
 *                o * 4 d + 256 h + 16 m + 2 i
 *   scales       token t = 8 o + i, group s of channels: bf16 at byte (o * d / group + s) * 16 + 2 i
 * (the orders in which the matrix instructions of the attention take them; 4.25 or 4.5 bits a value).
 * Quantiser, per token, head and `group` channels, all in FP32:
 *   x = float(k) - mean (mean = 0 where none is given);  a = max|x|;
 *   scale = a / 7 rounded UP to 5 significant bits;  nibble = 8 + rne(x / scale), 1 .. 15.
 *   a < 2^-100: scale 0, nibbles 8.  a >= 2^127, or an infinity or a NaN in the group: scale NaN, so that the group
 *   reads as NaN.
 * 5 bits of a scale times the 3 of a code fit the 8 of a bf16 number: what the cache holds is bf16 exactly, and no
 * kernel rounds it again.
 * Means: token means of K move its channel offsets out of the codes; the softmax does not see them (paper Sec. 3 "Q and K
 * Smoothing"), so the attention needs them for nothing and its LSE is the log-sum-exp of the smoothed logits, as
 * sagebwd_fwd's is.  V's mean is added back to O, the probabilities of a row summing to 1.  Both are float32 [H, d], or
 * NULL, and one for all tokens and requests of a call: a model's, measured once, with which the whole pool is filled.  (All
 * keys that a row sees need the same mean, whichever it is: means that differ between requests, as sagebwd_export_stats
 * gives them for one prompt, take an append for each request; V's take an attention for each, too.)
 *
 * Page numbers: a request's pages stand in its row of the block table, int32 [R, columns].  An entry outside
 * 0 .. pages - 1 stands for a page that does not exist: its tokens are not attended to.
 */
#ifndef SAGEBWD_SERVE_H
#define SAGEBWD_SERVE_H

#include "sagebwd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sagebwd_cache_params {
  int32_t H;      /* key/value heads */
  int32_t d;      /* 64 or 128 */
  int32_t page;   /* tokens of a page: 32, 64, 128 or 256 */
  int32_t group;  /* channels that share a scale: 32 or 64 */
  int32_t pages;  /* pages of the pool */
  int32_t reserved; /* must be 0 */
} sagebwd_cache_params;

/* Bytes of one page of the pool (all heads): H * page * (d + 4 d / group).  (`pages` is not looked at.) */
int sagebwd_cache_page_bytes(const sagebwd_cache_params* params, size_t* bytes);

/*
 * Pages, slots and positions of a step's new tokens.  Request r holds `held[r]` tokens and brings `added[r]` (0: none).
 * It needs need_r = ceil((held + added) / page) - ceil(held / page) new pages and is granted them if held, added >= 0,
 * held + added <= columns * page, its tokens are among the first `rows` of the step, and need_r is 0 or the sum of the
 * needs of the requests up to it is at most free_count.  The k-th page granted (requests in order, a request's pages in
 * order) is free_pages[free_count - 1 - k].  (Need that is not met counts all the same: behind a request for which there are not enough
 * pages none is granted a new one, so that a long request is not passed by short ones for ever.)
 *   block_table   int32 [R, columns], in and out: the granted pages go behind those that the request has
 *   free_pages    int32 [capacity], a stack; free_count int32 [1] (read as at most capacity)
 *   slots         int64 [rows]: page * (page number) + offset of every new token, requests in order; -1 for tokens of a
 *                 request that was not granted, and behind the last token
 *   positions     int32 [rows]: the token's place in its request (0 where the slot is -1 for those reasons)
 *   cu_new        int32 [R + 1]: where each request's tokens begin, and their end (a request whose sizes are not valid has
 *                 none; at most rows)
 *   lengths       int32 [R]: held + added, or held where not granted; may be `held`
 *   granted       int32 [R]: 1 or 0
 *   free_left     int32 [1]: free_count less the pages granted; may be `free_count`
 * Everything but block_table is out only, so that the call repeated on the same tensors does the same.
 * Bounds: R <= 2^20, columns * page < 2^30, R * columns < 2^31, rows <= 2^30.
 */
int sagebwd_cache_plan(const int32_t* held, const int32_t* added, int32_t* block_table, const int32_t* free_pages,
                       const int32_t* free_count, int32_t R, int32_t columns, int32_t page, int32_t capacity, int32_t rows,
                       int64_t* slots, int32_t* positions, int32_t* cu_new, int32_t* lengths, int32_t* granted, int32_t* free_left,
                       void* stream);

/*
 * The other way: request r keeps its first keep[r] tokens (0: it is done), and the pages that this frees go back on the
 * stack; the first request's first page is on top, so that trim after plan leaves the stack as it was.  lengths,
 * block_table (freed entries become -1), free_pages and free_count are changed in place.  A keep[r] outside 0 ..
 * lengths[r] leaves the request alone.  Entries that are not pages (negative) give none back.  (Pages beyond `capacity` are lost: the
 * stack has to hold every page.  A page that stands in two requests' rows comes back from each: who shares pages counts them and trims
 * the last one alone.)  Bounds as of plan.
 */
int sagebwd_cache_trim(const int32_t* keep, int32_t* lengths, int32_t* block_table, int32_t* free_pages, int32_t* free_count,
                       int32_t R, int32_t columns, int32_t page, int32_t capacity, void* stream);

/*
 * New keys and values into the cache, and what it holds out of it.  K, V: bf16 [T, H, d] with strides in elements
 * (multiples of 8; channels are adjacent; 16-byte aligned); slots int64 [T].  A slot outside the pool is skipped by
 * append and read as zeros.  Append wants every slot at most once (of tokens with one slot, any mixture stays).
 * read writes dense bf16 [T, H, d]: the values exactly, or with means value + mean in FP32, rounded to bf16.
 */
int sagebwd_cache_append(const void* K, const void* V, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                         int64_t v_head_stride, const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean,
                         const sagebwd_cache_params* params, void* pool, void* stream);
int sagebwd_cache_read(const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean, const sagebwd_cache_params* params,
                       const void* pool, void* K, void* V, void* stream);

typedef struct sagebwd_cache_call {
  int32_t R;          /* requests */
  int32_t T;          /* rows of Q and O (at least cu[R]; those behind it are left as they are).  From R * max_new on, with max_new * Hq / H
                         more than 32, the call takes every request to bring max_new tokens: shorter ones are slower than need be */
  int32_t Hq;         /* query heads: a multiple of H, at most 64 H; head h reads key/value head h / (Hq / H) */
  int32_t columns;    /* of the block table */
  int32_t max_new;    /* at least every request's new tokens (1: a decoding step); further tokens are not computed */
  int32_t max_length; /* at least every length, or 0: columns * page; a longer length is read as this.  Where the table is wider than the
                         requests are long it saves workspace, and a short batch the joining of parts */
  int32_t causal;     /* 1: new token i of n of a request of length L sees keys 0 .. i + L - n; 0: all L */
  float sm_scale;     /* 0 selects 1 / sqrt(d) */
  int64_t q_token_stride, q_head_stride; /* elements, multiples of 8; channels are adjacent */
} sagebwd_cache_call;

/*
 * Attention of every request's new tokens over its cache (which holds them already).
 *   Q           bf16 [T, Hq, d], strides as above, 16-byte aligned: row cu[r] + i is new token i of request r
 *   block_table int32 [R, columns]; lengths int32 [R] (tokens in the cache, the new ones among them); cu int32 [R + 1],
 *               rising from 0 (read as within 0 .. T)
 *   O           bf16 [T, Hq, d] dense; LSE float32 [Hq, T], or NULL
 * Sums, softmax statistics and the joining of parts are FP32; the probabilities times V's scales are rounded to bf16 for
 * the matrix instruction.  A row that sees no key (a request of length 0; with the mask the first rows of one shorter
 * than its new tokens; pages that do not exist) gives O = 0, LSE = -infinity.  What stands in the cache behind a
 * request's length reaches nothing.
 * Where max_new tokens are up to 32 query rows (new tokens x Hq / H) all requests go to a kernel for few rows, else to one for many; but where
 * T is less than R * max_new and Hq / H at most 32 the call launches both, and requests of up to 16 rows (32, where Hq / H is more than 16) go
 * to the former.  A tile of tokens on a page that does not exist is passed over by the kernel for few rows and masked by the others.
 * Where a call has few items for the machine their keys are divided over it and the parts joined by a further launch; from 2048 rows a request on, keys and values are
 * unpacked to bf16 in the workspace first (256 d bytes for 64 tokens and head; at most 4 GiB, else each tile unpacks its own).  How
 * work is divided depends on all requests of the call, so that O agrees between calls of different batches to its rounding, and bit
 * for bit between equal calls.
 * Range: with |Q| < 2^117, and V's largest magnitude (less its mean) times the request's length < 2^117, no sum overflows where the result does
 * not.  (Logits: nibbles are read as 16 .. 31 and 24 sum(Q) taken off.  Values: a row's sum is formed before it is divided, of probabilities
 * relative to a reference up to 2^8 below the largest, times nibbles of 31.)  Beyond it rows may be infinite or NaN.
 * The workspace depends on the host's sizes alone; its contents before the call do not matter, and calls in flight at a time (on two
 * streams, in two graphs) need one each.
 * Bounds: R <= 2^20, columns * page < 2^30, R * H * (columns * page / 128 + 3) <= 2^29, T * Hq / H < 2^30; with more than 32 rows a request
 * (T * Hq / H / 64 + R) * H <= 2^22.
 */
int sagebwd_cache_workspace_bytes(const sagebwd_cache_params* params, const sagebwd_cache_call* call, size_t* bytes);
int sagebwd_cache_attention(const void* Q, const void* pool, const int32_t* block_table, const int32_t* lengths, const int32_t* cu,
                            const float* v_mean, const sagebwd_cache_params* params, const sagebwd_cache_call* call, void* O, float* LSE,
                            void* workspace, size_t workspace_bytes, void* stream);

/* ---- rotary positions ------------------------------------------------------------------------------------------ */
typedef struct sagebwd_rotary_params {
  int32_t B, N;       /* tokens: B batches of N rows (packed tokens: B = 1) */
  int32_t Hq, Hk, d;  /* heads of Q and of K (Hk = 0: no K), d a multiple of 16 up to 512 */
  int32_t rotary_dim; /* channels that turn: a multiple of 16 up to d; the others are copied */
  int32_t axes;       /* 1 .. 4 (text: 1; video: time, height, width) */
  int32_t sections[4];/* frequencies of each axis, in order; their sum is rotary_dim / 2 */
  int32_t adjacent;   /* 0: channel i turns with i + rotary_dim / 2; 1: 2 i with 2 i + 1 */
  int32_t inverse;    /* 1: by the negative angle: the gradient of the call without it */
  int32_t positions64;/* 0: positions are int32, 1: int64 */
  int64_t q_strides[3], k_strides[3];   /* of the inputs: batch, row, head, in elements, multiples of 8 */
  int64_t qo_strides[3], ko_strides[3]; /* of the outputs */
} sagebwd_rotary_params;

/*
 * Rotary positions of Q and K: frequency i of a token turns (x1, x2) by theta = position[axis of i] * inv_freq[i]:
 *   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin.
 * positions [axes, B * N], inv_freq float32 [rotary_dim / 2].  The angle is formed and reduced in float64 (a float32 product loses
 * 0.06 rad at position 2^20), sine, cosine and the turn are FP32, the result is rounded once to bf16.  Outputs may be the
 * inputs (with the same strides).
 */
int sagebwd_rotary(const void* Q, const void* K, void* Qo, void* Ko, const void* positions, const float* inv_freq,
                   const sagebwd_rotary_params* params, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SAGEBWD_SERVE_H */
