/* cnnk_rel.h - C ABI of what a Vision Transformer block takes in beside cnnk_vit.h: dropout and stochastic depth from a
 * counter-based generator, and self-attention with a learned relative position bias, dropout of the probabilities, padded
 * batches, masked pairs and any number of tokens (gfx950 / MI355X).  Same conventions as cnnk.h and cnnk_vit.h: device
 * pointers and sizes, status codes of cnnk_status, nothing is allocated or synchronised, every call is enqueued on `stream`,
 * `dtype` names the storage type of activations and their gradients; parameters, their gradients and statistics are float.
 * Pointers to activations, to bias and to workspaces are 16-byte aligned, to `rng`, stats 8-byte, others to their element
 * (CNNK_ERR_UNSUPPORTED).  Results are reproducible bit for bit: no sum depends on the order in which workgroups run.
 */
#ifndef CNNK_REL_ABI_H_
#define CNNK_REL_ABI_H_
#include "cnnk.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- random numbers -----------------------------------------------------------------------------------------
 * A draw is a function of the state, the call's site and the element's place; nothing is stored, and the backward call forms
 * the same draws again.  The generator is Philox4x32 with seven rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel
 * random numbers: as easy as 1, 2, 3", SC 2011): F(c0, c1, c2, c3; k0, k1), four 32-bit words from four words and two of key.
 *   state  rng[2] in device memory: seed and step, 64 bits each.  The forward and the backward call of one training step read
 *          the same state; the program moves the step on between training steps (cnnk_rng_advance: a launch, so that a
 *          captured step draws anew at every replay).
 *   site   a number of the caller's for each call within a step (a layer): sites and steps draw independently.
 *   key    words 0 and 1 of F(step low, step high, site, 0; seed low, seed high)
 *   draw   a 16-bit piece of a word of F(...; key): an element is dropped if its draw is below round(65536 p).  Which
 *          one is said at each operator.  Kept values are divided by the exact share that is kept, 1 - round(65536 p) / 65536,
 *          within 7.7e-6 of 1 - p.
 * 0 <= p < 1 (CNNK_ERR_SHAPE otherwise); p so near 1 that nothing would be kept is CNNK_ERR_UNSUPPORTED.  Where round(65536 p) is 0,
 * rng is not read and may be NULL. */
int cnnk_rng_advance(unsigned long long* rng, unsigned long long by, void* stream);      /* step += by */

/* ---- dropout, with the bias in front of it and the residual sum behind it ------------------------------------------
 * y = res + keep * (z + bias) / (1 - p): fp32, rounded once.  bias [C] and res [rows][C] may be NULL.  span = 0: every element has
 * a draw of its own, element e = r * C + c the piece e % 8 (low halves first) of F(e / 8 low, e / 8 high, 0, 0).  span > 0: rows
 * i * span .. (i + 1) * span - 1 share one, the piece i % 8 of F(i / 8 low, i / 8 high, 0, 1) (stochastic depth: span = the
 * rows of an image).  z, res, y: [rows][C] of dtype; y may alias z or res.  C % 8 == 0. */
typedef struct { long long rows; int C; int dtype; float p; unsigned site; int span; } cnnk_dropout_desc;
int cnnk_dropout_fwd(const cnnk_dropout_desc* d, const void* z, const float* bias, const void* res,
                     const unsigned long long* rng, void* y, void* stream);

/* dz = keep * dy / (1 - p); dbias[c] = sum_r dz[r, c] of the unrounded values, if dbias is not NULL (the gradient of res is dy
 * itself).  dz may alias dy.  ws is needed with dbias only, C is 2^30 at most then. */
size_t cnnk_dropout_workspace_bytes(const cnnk_dropout_desc* d);
int cnnk_dropout_bwd(const cnnk_dropout_desc* d, const void* dy, const unsigned long long* rng, void* dz, float* dbias, void* ws,
                     size_t ws_bytes, void* stream);

/* ---- buckets of a relative position bias ----------------------------------------------------------------------------
 * bucket [T][T] int: the row of the bias table that query t takes for key u.  A number outside 0 .. buckets - 1 masks the pair.
 * cnnk_rel_buckets_grid writes that of a grid of gh x gw patches (T = gh * gw, row by row): the offset (yt - yu + gh - 1) *
 * (2 gw - 1) + xt - xu + gw - 1; with cls != 0 a class token in front of them has buckets n = (2 gh - 1)(2 gw - 1) (its keys
 * among the patches), n + 1 (it as a key) and n + 2 (itself).
 * cnnk_rel_plan lays a map out for the calls below (which pairs a bucket has, and the map in the order in which they read it).
 * A program makes a plan once for each map; `plan` is device memory of cnnk_rel_plan_bytes, 256-byte aligned.  It holds its T and buckets: a
 * call whose descriptor has others (its plan being memory of that many bytes all the same) gives NaN for every token and in all of dtable.
 * 1 <= T <= 8192, 1 <= buckets <= 16382. */
int cnnk_rel_buckets_grid(int gh, int gw, int cls, int* bucket, void* stream);
size_t cnnk_rel_plan_bytes(int T, int buckets);                  /* 0: unsupported */
size_t cnnk_rel_plan_workspace_bytes(int T, int buckets);
int cnnk_rel_plan(int T, int buckets, const int* bucket, void* plan, void* ws, size_t ws_bytes, void* stream);

/* ---- self-attention -----------------------------------------------------------------------------------------------------
 * qkv [B][T][3 * heads * dh] and o as in cnnk_attention_fwd.
 *   x[t, u] = q_t . k_u / sqrt(dh) + table[bucket[t, u]][h];  A = softmax of x over the keys that t sees;  o_t = sum_u keep * A[t, u] v_u / (1 - p)
 * t sees u if the pair is not masked and both are tokens of the image: lens [B] (int, NULL: T of each) is the number of each image's tokens, its first
 * ones (taken as 0 .. T).  A row that sees no key, and every row past the image's tokens, has o = 0 and no part in any gradient;
 * what qkv and d_o hold past an image's tokens, NaN too, is of no account.  Scores of -infinity from the table mask as well; the
 * lowest finite value does not (a row of nothing else is shared out evenly).  Features of an image's own tokens must be finite:
 * masked pairs are computed and left out.  A score that is NaN or +infinity (from a feature or the table that is not finite, or by overflow) is
 * handed on as NaN: to the rows that see it, their statistics and all gradients they take part in, and maybe to other rows of that image and
 * head; a score of -infinity masks its pair wherever it comes from.
 * table [buckets][heads] float; buckets = 0: no bias, table and plan are not read.
 * Dropout: query t, key u of (image b, head h) has half u % 2 of word t % 4 of F(u / 2, t / 4, b * heads + h, 2).
 * Training: stats [B][heads][T][2] receives a reference near each row's largest x and the logarithm of
 * sum_u exp(x - reference) (a row that sees no key: -infinity and 0);
 * NULL in evaluation.
 * dh in {16, 32, 64, 128}; T <= 16384, 8192 with buckets; heads <= 65535; the elements of an image's qkv take less than 2^31 bytes;
 * (B * heads + 8) * (T / 32, rounded up, + 7) < 2^26 (the threads of a launch). */
typedef struct { int B, T, heads, dh; int dtype; int buckets; float p; unsigned site; } cnnk_rel_desc;
int cnnk_rel_attention_fwd(const cnnk_rel_desc* d, const void* qkv, const float* table, const void* plan, const int* lens,
                           const unsigned long long* rng, void* o, float* stats, void* stream);

/* dqkv (all of it: zeros past an image's tokens) and dtable [buckets][heads] (overwritten; NULL: not formed).  o, stats: as the forward call left them, with the same lens, rng and plan.
 * The workspace holds three floats for each row, and 4 KB for each head and block of 32 x 32 pairs, as often as a head's images lie in different workgroups (1.6 GB for
 * 8 images of 4096 tokens, 12 heads); with dtable = NULL the rows alone, what the descriptor with buckets = 0 needs. */
size_t cnnk_rel_attention_workspace_bytes(const cnnk_rel_desc* d);
int cnnk_rel_attention_bwd(const cnnk_rel_desc* d, const void* qkv, const void* o, const void* d_o,
                           const float* table, const void* plan, const int* lens, const unsigned long long* rng,
                           const float* stats, void* dqkv, float* dtable, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
