/*
 * qkn_pages.h -- C ABI of libqkn, part 6: the book of a paged cache's pages on
 * the device, and copies of pages (AMD MI355X, gfx950).
 *
 * Which pages a sequence has, and how many sequences have a page, are arrays
 * that the device keeps and that no call brings to the host: a serving loop
 * that is captured in a graph takes pages for its new tokens, drops and forks
 * sequences and moves pages together while it is replayed. qkn_rope_cache and
 * qkn_attn read the same table and lengths. One book serves all layers: a page
 * number is a page of every layer's pools.
 *
 * Conventions are those of qkn.h (device pointers owned by the caller,
 * asynchronous on `stream`, validation before any HIP call, negative status
 * codes, n == 0 a no-op). Calls on one book, or on one cache, go one after the
 * other. Results do not depend on timing: pages are taken lowest number first,
 * in the order of the list.
 */
#ifndef QKN_PAGES_H
#define QKN_PAGES_H

#include <stdint.h>

#include "qkn.h"
#include "qkn_cache.h"
#include "qkn_cache4.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 *   refs       int32 [num_pages]: how many rows have the page; 0: it is free.
 *   table      int32 [rows, ld_table]: entry e of a row is the page that holds
 *              its tokens [e * page_size, (e + 1) * page_size). Entries past the
 *              row's last page are not used, and may be written.
 *   kv_len     int32 [rows]: a row's tokens, 0: an empty row.
 *   num_pages  0 to 2^24.
 *   rows       >= 0.
 *   ld_table   pages that a row can have; ld_table * page_size < 2^31.
 *   page_size  a power of two, 1 to 65536.
 * An empty book is zeros. Only a row's last page is partly full, and it has
 * that page alone: growing a row writes into no page that another row has.
 * Whatever the arrays hold, calls stay inside them: a length outside
 * [0, ld_table * page_size] makes the call refuse the row (free takes it as the
 * nearest of these), a page number outside [0, num_pages) is passed over.
 */
typedef struct qkn_pages {
  int32_t* refs;
  int32_t* table;
  int32_t* kv_len;
  int64_t num_pages;
  int64_t ld_table;
  int32_t rows;
  int32_t page_size;
} qkn_pages;

/* The most rows that one call may list. */
#define QKN_PAGES_MOST 1024

/*
 * count[i] more tokens for row which[i] (which NULL: row i), i < n, with the
 * pages that they need; and where the new tokens go, in the order of the list:
 *   slots  int64 [T] or NULL: page * page_size + row of each new token, as
 *          qkn_rope_cache takes it;
 *   pos    int32 [T] or NULL: its position in the sequence;
 *   done   int32 [n]: the row's tokens now, or -1: refused.
 * Refused, without a change to the row: a row outside the book, listed before in
 * the same call, with a malformed length, with count < 0 or more tokens than
 * ld_table pages hold; and, where free pages do not suffice, the first row that
 * does not get all of its pages and every later one that needs any. Tokens of a
 * refused row keep their places in slots and pos (-1 and 0), as do those behind
 * the last (T more than the counts' sum). Tokens beyond T get pages and are not
 * listed.
 */
int qkn_pages_grow(const qkn_pages* book, const int32_t* which, const int32_t* count, int32_t n, int64_t T,
                   int64_t* slots, int32_t* pos, int32_t* done, void* stream);

/*
 * Row to[i] becomes a copy of row from[i], i < n: it shares the whole pages, and
 * has a page of its own for the last one where that is partly full. src[i] and
 * dst[i] (int32 [n]) are that page of from[i] and of to[i], for qkn_pages_copy, or
 * -1: nothing to copy. done (int32 [n]): the row's tokens, or -1: refused, namely
 * rows outside the book, a `to` that is not empty or listed before in the same
 * call, a malformed length of `from`, and pages as for qkn_pages_grow. Lengths
 * are those before the call, so a row that is empty then forks as an empty row.
 */
int qkn_pages_fork(const qkn_pages* book, const int32_t* from, const int32_t* to, int32_t n, int32_t* src,
                   int32_t* dst, int32_t* done, void* stream);

/*
 * Empties the rows which[i] (NULL: row i), i < n; pages that no row has any more
 * are free. Rows outside the book and rows listed again are passed over.
 */
int qkn_pages_free(const qkn_pages* book, const int32_t* which, int32_t n, void* stream);

/*
 * Moves pages in use to the front: the last page in use to the first free one,
 * the second last to the second, and so on while that is a move down, n moves at
 * most. src and dst (int32 [n]) are the moves, -1 behind the last one, for
 * qkn_pages_copy, which has to run before anything else uses the pages. No page
 * of dst is one of src. Table and refs are written to `out`, a book of the same
 * sizes (its kv_len is not used), or NULL: in place. The workspace is the call's
 * own while it runs.
 */
int64_t qkn_pages_compact_workspace_bytes(const qkn_pages* book);
int qkn_pages_compact(const qkn_pages* book, const qkn_pages* out, int32_t* src, int32_t* dst, int32_t n,
                      void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Copies page src[i] to page dst[i], i < n, K and V (and exponents), in each of
 * the `count` caches (an array on the host: the layers'). Pairs that are equal, or
 * of which one is outside [0, num_pages), are passed over. What a page holds that
 * is a pair's dst and another pair's src or dst is undefined. Caches may differ in
 * sizes and format; scales of FP8 caches are per head and stay.
 */
int qkn_pages_copy(const qkn_cache* caches, int32_t count, const int32_t* src, const int32_t* dst, int32_t n,
                   void* stream);
int qkn_pages_copy4(const qkn_cache4* caches, int32_t count, const int32_t* src, const int32_t* dst, int32_t n,
                    void* stream);

/*
 * All: QKN_EINVAL: a NULL or malformed book or cache, n, T or count < 0, NULL
 * arrays (which, slots and pos apart) where n > 0; a workspace that is NULL or
 * too small; an `out` of other sizes. QKN_EOVERLAP: an output array overlapping
 * another array of the call (compact: out's table and refs may be the book's), or
 * a pool. QKN_ENOTSUP: n over QKN_PAGES_MOST (grow, fork, free) or 2^24 (compact,
 * copy), more work than one grid holds, a workspace not 16-byte aligned.
 */

#ifdef __cplusplus
}
#endif

#endif /* QKN_PAGES_H */
