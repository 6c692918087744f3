/*
 * The books of a paged cache (autochunk_decode.h) behind the same library: which pages are in use and whose, pages freed and taken as sequences
 * grow, end and leave what their windows no longer see, sequences that go on as copies of others, and pages moved to the front.  All of it on
 * the device, in order of the stream, so that a step never waits for the host.  The conventions are those of autochunk_rt.h: nothing is allocated,
 * kept or synchronised.  Results do not depend on timing.
 */
#ifndef AUTOCHUNK_PAGES_H
#define AUTOCHUNK_PAGES_H

#include <stdint.h>

#include "autochunk_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * uses[p] is the number of places of page tables that name page p; a page with 0 (or less) is free.  A caller that keeps a page for itself, to share a prefix
 * for instance, adds one of its own.  Place i of sequence b, page_table[b * ld_page_table + i], is where tokens i * page up to (i + 1) * page - 1 lie; a number outside
 * [0, pages) names no page (-1 by these calls).  One set of books serves all layers: caches of the same pages.  pages at most 2^24, batch 65535, tokens of a sequence
 * (ld_page_table times page) and entries of a table (batch times ld_page_table) 2^30, else AC_ERR_UNSUPPORTED; arrays on 4-byte boundaries, page a multiple of 16.
 *
 * Every call reads the books `from` and leaves those after it in `to`, of the same sizes; each of `to`'s arrays may be `from`'s own (where a call does not say
 * otherwise) or lies apart from both of them.  What a call reads besides (ranges, parents, lengths) lies apart from the books `to`, what it leaves besides (lengths, numbers) from all books
 * and from everything else, else AC_ERR_ARG; all on 4-byte boundaries, else AC_ERR_ALIGN.  workspace: dev, 16-byte aligned, ac_pages_workspace_bytes() large, else AC_ERR_WORKSPACE; what it holds does not matter.
 */
typedef struct ac_page_books {
  int32_t* uses;                    /* dev, [pages] */
  int32_t* page_table;              /* dev, [batch][ld_page_table] */
  int64_t pages, ld_page_table, batch;
  int32_t page;                     /* tokens */
} ac_page_books;
uint64_t ac_pages_workspace_bytes(const ac_page_books* books);

/*
 * Frees pages, then takes others.  Of sequence b, places whose tokens all lie in [drop_begin[b], drop_end[b]) give up their pages: uses is one less, the place names
 * none.  Then places that have a token in [take_begin[b], take_end[b]) and name no page get one each, with uses 1: the free pages with the lowest numbers, the lowest one for the
 * first such place of the first sequence, and so on; pages that this call freed among them.  Where pages run out the other places name none.  drop_* and take_*: dev, [batch], each pair NULL where
 * nothing is freed or taken; tokens before 0 and behind the table count as no place's.  missing (dev, may be NULL) receives the number of places that got no page.
 */
int ac_op_pages_update(const ac_page_books* from, const ac_page_books* to, const int32_t* drop_begin, const int32_t* drop_end, const int32_t* take_begin,
                       const int32_t* take_end, int32_t* missing, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * Sequences go on as others: sequence j becomes a copy of sequence parent[j] as it was, of length[parent[j]] tokens, or, with a parent outside [0, batch), one without
 * tokens and pages; its length goes to length_to[j].  Pages whose tokens all belong to the sequence are shared.  What lies behind them, a page that is partly filled and
 * places for tokens to come, stays with the first sequence that has this parent; the others get a page of their own for the partly filled one, into which all caches' codes and scales of
 * its blocks are copied, and no places for tokens to come.  Pages that no place names any more are free, and serve these copies.  Which pages are taken, and what
 * happens where they run out, is as in ac_op_pages_update (the place names none: what it held is lost to that sequence).
 * A length that was set back below pages that others name, too, is the caller's matter: neither this call nor an update takes such pages from a sequence that goes on to write into them (first give them up,
 * ac_op_pages_update, and copy the partly filled one, ac_op_cache_copy_pages).
 * caches: the layers' caches, host array of n_caches (at most 4096; NULL with 0).  page_table of `to` and length_to lie apart from those of `from`.
 */
int ac_op_cache_fork(const ac_kv_cache* caches, int n_caches, const ac_page_books* from, const ac_page_books* to, const int32_t* parent, const int32_t* length,
                     int32_t* length_to, int32_t* missing, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * Moves pages in use to the front: with n of them, they are pages 0 .. n - 1 afterwards and those behind are free.  The last page in use goes to the first free one, and so
 * on, in all caches; uses and page tables follow (a page that a caller keeps for itself moves, too: its number is known where a row of the table names it).  used (dev, may be NULL) receives n.
 */
int ac_op_cache_compact(const ac_kv_cache* caches, int n_caches, const ac_page_books* from, const ac_page_books* to, int32_t* used, void* workspace,
                        uint64_t workspace_bytes, void* stream);

/*
 * Page target[i] becomes a copy of page source[i], in all caches: of its first tokens[i] tokens, in whole blocks of 16, or (tokens NULL) of all.  Pairs of which one names no page, or both the
 * same, are left out.  No page may be target of two pairs, or target of one and source of another.  source, target, tokens: dev, [n], on 4-byte boundaries, else AC_ERR_ALIGN, n at most 2^24.  The caches have the same pages.
 */
int ac_op_cache_copy_pages(const ac_kv_cache* caches, int n_caches, const int32_t* source, const int32_t* target, const int32_t* tokens, int64_t n,
                           void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AUTOCHUNK_PAGES_H */
