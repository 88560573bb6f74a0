// Host logic of the rotary embedding and the 8-bit cache: descriptor validation and launch planning.  Plain C++ like
// ta_host.cpp, and built with it everywhere.  See include/treeattn.h for the contract of every entry point.
#include <initializer_list>
#include <limits.h>
#include <math.h>
#include <string.h>

#include "ta_params.h"

namespace {

bool strides_given(const ta_tensor *t, bool unit_rows)
{
    for (int i = 0; i < t->ndim; ++i)
        if (t->stride[i] < 0)
            return false;
    return !unit_rows || t->stride[t->ndim - 1] == 1 || t->shape[t->ndim - 1] <= 1;
}

// No two elements of a tensor that is written at one address, as far as a stride of zero makes it so.
bool no_zero_stride(const ta_tensor *t)
{
    for (int i = 0; i < t->ndim; ++i)
        if (t->shape[i] > 1 && t->stride[i] == 0)
            return false;
    return true;
}

// Do all rows start on 16 bytes?  (A dimension of extent 1 has no stride that counts.)
bool on_16_bytes(const ta_tensor *t)
{
    const int64_t per16 = t->dtype == TA_E4M3 ? 16 : t->dtype == TA_BF16 ? 8 : 4;
    if ((uintptr_t)t->data % 16 != 0)
        return false;
    for (int i = 0; i < t->ndim - 1; ++i)
        if (t->shape[i] > 1 && t->stride[i] % per16 != 0)
            return false;
    return true;
}

int check_rows(const ta_tensor *t, int32_t dtype, int64_t B, int64_t T, int64_t H, int64_t D, bool written)
{
    if (t->dtype != dtype)
        return TA_ERR_DTYPE;
    if (t->ndim != 4)
        return TA_ERR_RANK;
    if (t->shape[0] != B || t->shape[1] != T || t->shape[2] != H || t->shape[3] != D)
        return TA_ERR_SHAPE;
    if (!strides_given(t, true) || (written && !no_zero_stride(t)))
        return TA_ERR_STRIDE;
    return B > 0 && !t->data ? TA_ERR_NULL : TA_OK;
}

struct Cache {
    int64_t n_pages, Hkv, ps, D, capacity;
};

// Caches, scales and page table of B requests.
int check_cache(const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs, const ta_tensor *pt, int64_t B,
                bool written, Cache *c)
{
    for (const ta_tensor *t : {k, v})
        if (t->dtype != TA_E4M3)
            return TA_ERR_DTYPE;
    for (const ta_tensor *t : {ks, vs})
        if (t->dtype != TA_E8M0)
            return TA_ERR_DTYPE;
    if (pt && pt->dtype != TA_I32)
        return TA_ERR_DTYPE;
    if (k->ndim != 4 || v->ndim != 4 || ks->ndim != 3 || vs->ndim != 3 || (pt && pt->ndim != 2))
        return TA_ERR_RANK;
    c->n_pages = k->shape[0]; c->Hkv = k->shape[1]; c->ps = k->shape[2]; c->D = k->shape[3];
    if (c->D < 1 || c->D > TA_MAX_HEAD_DIM)
        return TA_ERR_HEAD_DIM;
    if (c->Hkv < 1)
        return TA_ERR_HEADS;
    if (c->n_pages < 0 || c->n_pages > INT32_MAX || c->ps < 1 || c->ps > (1 << 30) || c->Hkv > 65535)
        return TA_ERR_SHAPE;
    for (int i = 0; i < 4; ++i)
        if (v->shape[i] != k->shape[i])
            return TA_ERR_SHAPE;
    for (int i = 0; i < 3; ++i)
        if (ks->shape[i] != k->shape[i] || vs->shape[i] != k->shape[i])
            return TA_ERR_SHAPE;
    if (pt ? (pt->shape[0] != B || pt->shape[1] < 1) : c->n_pages < B)
        return TA_ERR_PAGE_TABLE;
    if (pt && pt->shape[1] > INT32_MAX)
        return TA_ERR_SHAPE;
    if (!strides_given(k, true) || !strides_given(v, true) || !strides_given(ks, false) || !strides_given(vs, false) ||
        (pt && !strides_given(pt, true)))
        return TA_ERR_STRIDE;
    if (written && (!no_zero_stride(k) || !no_zero_stride(v) || !no_zero_stride(ks) || !no_zero_stride(vs)))
        return TA_ERR_STRIDE;
    c->capacity = pt ? pt->shape[1] * c->ps : c->ps;
    if (c->capacity > INT32_MAX)
        return TA_ERR_SHAPE;
    if (B > 0)
        for (const ta_tensor *t : {k, v, ks, vs})
            if (!t->data)
                return TA_ERR_NULL;
    return B > 0 && pt && !pt->data ? TA_ERR_NULL : TA_OK;
}

int check_lens(const ta_tensor *sl, int64_t B)
{
    if (sl->dtype != TA_I32)
        return TA_ERR_DTYPE;
    if (sl->ndim != 1)
        return TA_ERR_RANK;
    if (sl->shape[0] != B)
        return TA_ERR_SHAPE;
    if (sl->stride[0] < 0)
        return TA_ERR_STRIDE;
    return B > 0 && !sl->data ? TA_ERR_NULL : TA_OK;
}

// Frequencies, tree and options of a call that rotates rows [B, T, H, D].
int check_turn(const ta_tensor *freqs, const ta_tensor *par, const ta_rope_opts *o, int64_t B, int64_t T, int64_t D, TARows *r)
{
    if (freqs->dtype != TA_F32 || (par && par->dtype != TA_I32))
        return TA_ERR_DTYPE;
    if (freqs->ndim != 1 || (par && par->ndim != 1 && par->ndim != 2))
        return TA_ERR_RANK;
    if (freqs->shape[0] < 1 || 2 * freqs->shape[0] > D)
        return TA_ERR_SHAPE;
    if (par) {
        if (T > TA_MAX_TREE)
            return TA_ERR_TREE_SIZE;
        if (par->shape[par->ndim - 1] != T || (par->ndim == 2 && par->shape[0] != B))
            return TA_ERR_SHAPE;
        if (!strides_given(par, true))
            return TA_ERR_STRIDE;
    }
    if (!strides_given(freqs, true))
        return TA_ERR_STRIDE;
    if (B > 0 && (!freqs->data || (par && !par->data)))
        return TA_ERR_NULL;
    r->amplitude = 1.f;
    if (o) {
        if ((o->interleaved != 0 && o->interleaved != 1) || !(o->amplitude >= 0.f) || !isfinite(o->amplitude))
            return TA_ERR_OPTS;
        if (o->tree_masks && (!par || ((uintptr_t)o->tree_masks % 8) != 0 || o->tree_masks_stride < 0))
            return TA_ERR_OPTS;
        if (o->status && ((uintptr_t)o->status % 4) != 0)
            return TA_ERR_OPTS;
        r->interleaved = o->interleaved;
        if (o->amplitude > 0.f)
            r->amplitude = o->amplitude;
        r->masks_in = (const unsigned long long *)o->tree_masks;
        r->masks_sb = o->tree_masks_stride;
        r->status2 = o->status;
    }
    r->freqs = (const float *)freqs->data;
    r->R = (int)(2 * freqs->shape[0]);
    r->parent = par ? (const int32_t *)par->data : nullptr;
    r->par_sb = par && par->ndim == 2 ? par->stride[0] : 0;
    return TA_OK;
}

// An output may be its input itself, element for element, and must not start there otherwise.
int check_in_place(const ta_tensor *in, const ta_tensor *out)
{
    if (in->data != out->data)
        return TA_OK;
    for (int i = 0; i < 4; ++i)
        if (in->shape[i] > 1 && in->stride[i] != out->stride[i])
            return TA_ERR_STRIDE;
    return TA_OK;
}

int check_step(int64_t B, int64_t T, int64_t D, int64_t Hq, int64_t Hkv)
{
    if (B < 0 || B > TA_MAX_BATCH)
        return TA_ERR_BATCH;
    if (T < 1)
        return TA_ERR_TREE_SIZE;
    if (T > INT32_MAX)
        return TA_ERR_SHAPE;
    if (D < 1 || D > TA_MAX_HEAD_DIM)
        return TA_ERR_HEAD_DIM;
    if (Hq < 0 || Hkv < 0 || Hq > 65535 || Hkv > 65535)
        return TA_ERR_SHAPE;
    return TA_OK;
}

void set_cache(const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs, const ta_tensor *pt,
               const Cache &c, TARows *r)
{
    r->kc = k->data; r->vc = v->data;
    r->ks = (uint8_t *)ks->data; r->vs = (uint8_t *)vs->data;
    r->k_sp = k->stride[0]; r->k_shc = k->stride[1]; r->k_ss = k->stride[2];
    r->v_sp = v->stride[0]; r->v_shc = v->stride[1]; r->v_ss = v->stride[2];
    r->ks_sp = ks->stride[0]; r->ks_sh = ks->stride[1]; r->ks_ss = ks->stride[2];
    r->vs_sp = vs->stride[0]; r->vs_sh = vs->stride[1]; r->vs_ss = vs->stride[2];
    r->page_table = pt ? (const int32_t *)pt->data : nullptr;
    r->pt_sb = pt ? pt->stride[0] : 0;
    r->ps = (int)c.ps; r->capacity = (int)c.capacity; r->n_pages = (int)c.n_pages;
}

// Tokens that a workgroup takes: one, until there are several workgroups per compute unit, whose start then counts more than
// what one has to do (a prompt of 8000 tokens with 40 heads).
int tokens_per_group(int64_t tokens_all, int64_t rows_per_token, int most = 8, int rows = 128)
{
    int n = 1;
    while (n < most && tokens_all / (2 * n) >= 4 * 256 && rows_per_token * n < rows)
        n *= 2;
    return n;
}

// The launch plan of the matrix-core kernel, over that of the scalar one, whose checks have been made.
int plan_mfma(const ta_tensor *out, const ta_opts *opts, int num_cus, TAProblem *pr)
{
    TAParams &p = pr->p;
    TAPlan &pl = pr->plan;
    const int num_splits = opts ? opts->num_splits : 0, item_cost = opts ? opts->item_cost : 0;
    const int64_t lists = (int64_t)p.B * p.Hkv, l1 = lists > 0 ? lists : 1;
    const int64_t tiles_cap = lists * ((p.capacity - p.T + TA_TILE - 1) / TA_TILE + 1);
    pl.kernel = TA_KERNEL_MFMA;
    // Query rows of a workgroup.  Up to 32 have a kernel of their own (ta_q8_attn.hip: every wave for itself).  More of them
    // take tiles of 64, 128 or 256 rows, those that cost least: a pass over the keys takes 109, 179 and 302, relative to one another
    // (256 rows, 4 requests of 131072 tokens: 872, 714 and 604 us, and 961 in blocks of 32; 320 rows, 8 requests of 32768: 540, 504 and
    // 550; 64 rows, 32 requests of 512 to 8192 tokens: 80, 110 and 168 us, and 101).
    const int sizes[3] = {64, 128, 256}, costs[3] = {109, 179, 302};
    p.ks_rows = p.is_bf16 ? 32 : 128;
    for (int64_t i = 0, least = INT64_MAX; p.is_bf16 && p.rows > 32 && i < 3; ++i) {
        const int64_t cost = (int64_t)((p.rows + sizes[i] - 1) / sizes[i]) * costs[i];
        if (cost < least) {
            least = cost;
            p.ks_rows = sizes[i];
        }
    }
    // (fp32 queries, each the sum of three bf16 numbers, have blocks of 128 rows: 128 requests with 8 rows and 8192 tokens 120 us, and
    // 1670 with the scalar kernel; 32 requests with 64 rows, 8 KV heads, 4096 tokens 130 and 6540)
    pl.ks_rows = p.ks_rows;
    p.basic = p.ks_rows == 32;
    const int blocks = (p.rows + p.ks_rows - 1) / p.ks_rows;
    p.rows_grp = pl.rows_grp = p.rows;
    p.n_rg = pl.n_rg = 1;
    // (what a share of a list costs beside its tiles: 128 requests of 8 KV heads, one new token, 15 105 us, 9 117; 20 costs 1 % more.
    // With tiles for all waves 9 to 13 are the same within 2 %.)
    pl.item_cost = item_cost > 0 ? item_cost : lists == 1 ? 6 : p.basic ? 15 : 9;
    p.pad = pl.item_cost - 1;
    if (tiles_cap + lists * p.pad > INT32_MAX)
        return TA_ERR_SHAPE;
    // Workgroups of four waves, two on a compute unit, wait for one another less, and take more shares, each with its start and its
    // partial results: 64 rows, 64 requests of 8 KV heads, 512 to 4096 tokens 52 us, 60 with eight waves; 32 of 512 to 8192: 84 and
    // 88; but 8 of 4096: 31 and 29, and 128 rows in one request of 8192: 34 and 31.  With no more tiles than workgroups every share is one
    // of the smaller tiles: 64 rows in one list of 8192 tokens 16.4 us, 18.1 with eight waves, 8 lists of 2048 17.7 and 19.5; 16 of 2000, which
    // are past the line, 20.0 and 19.9.  (Up to 32 rows: 128 requests, one new token 112 us,
    // 105 with eight waves.)
    const bool small_blocks = p.is_bf16 && (p.ks_rows == 64 || p.ks_rows == 128);
    const bool pairs = small_blocks && (tiles_cap >= 64 * (int64_t)num_cus || tiles_cap <= num_cus + num_cus / 4);
    pl.threads = pairs ? 256 : 512;
    int64_t want = (pairs ? 2 : 1) * num_cus / blocks;
    if (blocks > 1 && want > 8)
        want -= want % 8;                                   // (blocks of the same keys on one XCD, where the L2 has them for all but the first)
    pl.n_wg = (int)(num_splits > 0 ? num_splits : want > 0 ? want : 1);
    if (pl.n_wg > tiles_cap)
        pl.n_wg = (int)(tiles_cap > 0 ? tiles_cap : 1);
    p.n_wg = pl.n_wg;
    p.min_q = pl.min_q = 1;
    pl.n_slots = pl.n_wg + (int)lists;
    const bool out_aligned = ((uintptr_t)out->data % 16) == 0 && p.o_sb % 4 == 0 && p.o_st % 4 == 0 && p.o_sh % 4 == 0;
    const int64_t parts = (pl.n_wg + l1 - 1) / l1 + 1;
    p.merge_kind = !out_aligned ? TA_MERGE_GENERAL : parts >= 13 && lists * p.rows <= 1024 ? TA_MERGE_WIDE : TA_MERGE_ROW;
    p.part_q15 = p.is_bf16;                                // (fp32 queries keep fp32 partial results)
    p.ls = p.is_bf16 ? 2 : 1;
    p.one_parts = 0;
    if (lists == 1 && num_splits == 0 && p.merge_kind == TA_MERGE_WIDE && pl.n_wg > 8192 / p.D)
        p.one_parts = 8192 / p.D;
    pl.merge_kind = p.merge_kind;
    const int mrows = ta_host_merge_rows(p);
    pl.merge_wgs = (int)lists * ((p.rows + mrows - 1) / mrows);
    const size_t rows_total = (size_t)pl.n_slots * p.rows_grp;
    pr->ws_o_bytes = ta_host_align_up(rows_total * p.D * sizeof(float), 256);
    pr->ws_lse_bytes = ta_host_align_up(rows_total * sizeof(float), 256);
    pr->ws_ls_off = p.part_q15 ? ta_host_align_up(rows_total * p.D * 2, 256) : pr->ws_o_bytes;
    pr->ws_bytes = pr->ws_o_bytes + pr->ws_lse_bytes + ta_host_align_up((size_t)lists * 2 * sizeof(int32_t), 256);
    // Short lists go to one workgroup each, which writes the outputs itself: no schedule, no partial results, no merge pass.  Up to
    // how many tiles depends on what a tile takes the workgroup, and on how many stand idle meanwhile (tokens, us uncut / cut):
    //     rows        8 lists                64 lists               256 lists
    //     32          1024  13.2/13.3        1024  14.0/16.9        1024  16.6/22.0
    //                 1536  16.0/13.3        1536  16.6/16.5        2048  26.3/31.9
    //     64           256  14.0/15.9         512  18.3/19.3        1024  27.2/30.9
    //                  512  17.8/16.1         768  21.8/19.5        2048  42.1/43.0
    //     256          128  21.8/26.5         256  27.1/29.8        1024  60.3/72.9
    //                  256  26.5/25.4         768  44.5/33.2        2048  96.7/105.6
    //     fp32         256  16.5/17.5         256  16.9/20.1        1024  38.9/41.5
    //                  768  38.2/16.6         768  38.5/27.1        1536  52.7/54.1
    // (A batch of uneven lengths waits for its longest list: the line for a full chip stays where the gain is a tenth and more.)
    // More lists than workgroups run at a time take rounds, the last of which may be almost empty.  In tiles, a round takes some 10 and
    // the list's (8 with two workgroups on a compute unit); cut, a list takes some 15 (20) and its own, and the call 6: 64 rows, 2048 lists
    // of 200 tokens 68 us uncut, 134 cut, 640 lists of 1000 60 and 74; 256 rows, 400 lists of 500 tokens 77 and 90, 264 lists (two rounds for
    // eight of them) of 1000 106 and 83.
    const int64_t groups = lists * blocks, n = lists > 0 ? tiles_cap / lists : 0;
    const int64_t slots = groups <= num_cus ? num_cus : (p.basic || small_blocks ? 2 : 1) * (int64_t)num_cus;
    const int64_t rounds = (groups + slots - 1) / slots;
    const int64_t solo_start = slots > num_cus ? 8 : 10, cut_start = slots > num_cus ? 20 : 15;
    const int line = 4 * groups >= 3 * slots ? 32 : p.basic || groups > num_cus ? 18 : p.ks_rows == 64 ? 8 : 5;
    if (num_splits == 0 && item_cost == 0 && lists > 0 && p.merge_kind != TA_MERGE_GENERAL && n <= line &&
        (rounds == 1 || rounds * (n + solo_start) * slots <= 6 * slots + groups * (n + cut_start)))
        p.solo = slots == num_cus ? TA_SOLO_WIDE : TA_SOLO_PAIR;
    if (p.solo)
        pl.merge_wgs = 0;
    return TA_OK;
}

}  // namespace

int ta_host_check_rope(const ta_tensor *q, const ta_tensor *k, const ta_tensor *freqs, const ta_tensor *sl, const ta_tensor *par,
                       const ta_tensor *qo, const ta_tensor *ko, const ta_rope_opts *opts, TARows *r)
{
    if (!q || !freqs || !sl || !qo || (k != nullptr) != (ko != nullptr))
        return TA_ERR_NULL;
    if (q->dtype != TA_BF16 && q->dtype != TA_F32)
        return TA_ERR_DTYPE;
    if (q->ndim != 4 || (k && k->ndim != 4))
        return TA_ERR_RANK;
    const int64_t B = q->shape[0], T = q->shape[1], Hq = q->shape[2], D = q->shape[3], Hkv = k ? k->shape[2] : 0;
    int rc = check_step(B, T, D, Hq, Hkv);
    if (rc != TA_OK)
        return rc;
    if (Hq < 1 || (k && Hkv < 1))
        return TA_ERR_HEADS;
    memset(r, 0, sizeof *r);
    if ((rc = check_rows(q, q->dtype, B, T, Hq, D, false)) != TA_OK || (rc = check_rows(qo, q->dtype, B, T, Hq, D, true)) != TA_OK ||
        (k && (rc = check_rows(k, q->dtype, B, T, Hkv, D, false)) != TA_OK) ||
        (k && (rc = check_rows(ko, q->dtype, B, T, Hkv, D, true)) != TA_OK) || (rc = check_lens(sl, B)) != TA_OK ||
        (rc = check_turn(freqs, par, opts, B, T, D, r)) != TA_OK || (rc = check_in_place(q, qo)) != TA_OK ||
        (k && (rc = check_in_place(k, ko)) != TA_OK))
        return rc;
    r->q = q->data; r->q_out = qo->data;
    r->q_sb = q->stride[0]; r->q_st = q->stride[1]; r->q_sh = q->stride[2];
    r->qo_sb = qo->stride[0]; r->qo_st = qo->stride[1]; r->qo_sh = qo->stride[2];
    if (k) {
        r->k = k->data; r->k_out = ko->data;
        r->k_sb = k->stride[0]; r->k_st = k->stride[1]; r->k_sh = k->stride[2];
        r->ko_sb = ko->stride[0]; r->ko_st = ko->stride[1]; r->ko_sh = ko->stride[2];
    }
    r->seq_lens = (const int32_t *)sl->data;
    r->sl_s = sl->stride[0];
    r->B = (int)B; r->T = (int)T; r->Hq = (int)Hq; r->Hkv = (int)Hkv; r->D = (int)D;
    r->capacity = INT32_MAX;
    r->is_bf16 = q->dtype == TA_BF16;
    r->vec = D % 16 == 0 && r->R % 16 == 0 && on_16_bytes(q) && on_16_bytes(qo) && (!k || (on_16_bytes(k) && on_16_bytes(ko)));
    r->tokens = tokens_per_group(B * T, Hq + Hkv);
    return TA_OK;
}

int ta_host_check_q8_append(const ta_tensor *kn, const ta_tensor *vn, const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks,
                            const ta_tensor *vs, const ta_tensor *pt, const ta_tensor *sl, TARows *r)
{
    if (!kn || !vn || !k || !v || !ks || !vs || !sl)
        return TA_ERR_NULL;
    if (kn->dtype != TA_BF16 && kn->dtype != TA_F32)
        return TA_ERR_DTYPE;
    if (kn->ndim != 4)
        return TA_ERR_RANK;
    const int64_t B = kn->shape[0], T = kn->shape[1], Hkv = kn->shape[2], D = kn->shape[3];
    int rc = check_step(B, T, D, 0, Hkv);
    if (rc != TA_OK)
        return rc;
    Cache c;
    if ((rc = check_cache(k, v, ks, vs, pt, B, true, &c)) != TA_OK || (rc = check_rows(kn, kn->dtype, B, T, c.Hkv, c.D, false)) != TA_OK ||
        (rc = check_rows(vn, kn->dtype, B, T, c.Hkv, c.D, false)) != TA_OK || (rc = check_lens(sl, B)) != TA_OK)
        return rc;
    if (c.capacity < T)
        return TA_ERR_PAGE_TABLE;
    memset(r, 0, sizeof *r);
    r->k = kn->data; r->v = vn->data;
    r->k_sb = kn->stride[0]; r->k_st = kn->stride[1]; r->k_sh = kn->stride[2];
    r->v_sb = vn->stride[0]; r->v_st = vn->stride[1]; r->v_sh = vn->stride[2];
    set_cache(k, v, ks, vs, pt, c, r);
    r->seq_lens = (const int32_t *)sl->data;
    r->sl_s = sl->stride[0];
    r->B = (int)B; r->T = (int)T; r->Hkv = (int)Hkv; r->D = (int)D;
    r->amplitude = 1.f;
    r->is_bf16 = kn->dtype == TA_BF16;
    r->vec = D % 16 == 0 && on_16_bytes(kn) && on_16_bytes(vn) && on_16_bytes(k) && on_16_bytes(v);
    r->tokens = tokens_per_group(B * T, 2 * Hkv);
    return TA_OK;
}

int ta_host_check_q8_rope_append(const ta_tensor *q, const ta_tensor *kn, const ta_tensor *vn, const ta_tensor *freqs,
                                 const ta_tensor *sl, const ta_tensor *par, const ta_tensor *qo, const ta_tensor *k,
                                 const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs, const ta_tensor *pt,
                                 const ta_rope_opts *opts, TARows *r)
{
    if (!q || !qo || !freqs)
        return TA_ERR_NULL;
    int rc = ta_host_check_q8_append(kn, vn, k, v, ks, vs, pt, sl, r);
    if (rc != TA_OK)
        return rc;
    if (q->ndim != 4)
        return TA_ERR_RANK;
    const int64_t Hq = q->shape[2];
    if (Hq < 1)
        return TA_ERR_HEADS;
    if (Hq > 65535)
        return TA_ERR_SHAPE;
    if ((rc = check_rows(q, kn->dtype, r->B, r->T, Hq, r->D, false)) != TA_OK ||
        (rc = check_rows(qo, kn->dtype, r->B, r->T, Hq, r->D, true)) != TA_OK ||
        (rc = check_turn(freqs, par, opts, r->B, r->T, r->D, r)) != TA_OK || (rc = check_in_place(q, qo)) != TA_OK)
        return rc;
    r->q = q->data; r->q_out = qo->data;
    r->q_sb = q->stride[0]; r->q_st = q->stride[1]; r->q_sh = q->stride[2];
    r->qo_sb = qo->stride[0]; r->qo_st = qo->stride[1]; r->qo_sh = qo->stride[2];
    r->Hq = (int)Hq;
    r->vec = r->vec && r->R % 16 == 0 && on_16_bytes(q) && on_16_bytes(qo);
    r->tokens = tokens_per_group((int64_t)r->B * r->T, Hq + 2 * r->Hkv);
    return TA_OK;
}

int ta_host_check_q8_read(const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs, const ta_tensor *pt,
                          const ta_tensor *starts, const ta_tensor *counts, const ta_tensor *ko, const ta_tensor *vo, TAQ8Read *r)
{
    if (!k || !v || !ks || !vs || !counts || !ko || !vo)
        return TA_ERR_NULL;
    if (ko->dtype != TA_BF16 && ko->dtype != TA_F32)
        return TA_ERR_DTYPE;
    if (ko->ndim != 4)
        return TA_ERR_RANK;
    const int64_t B = ko->shape[0], N = ko->shape[1];
    if (B < 0 || B > TA_MAX_BATCH)
        return TA_ERR_BATCH;
    if (N < 0 || N > INT32_MAX)
        return TA_ERR_SHAPE;
    Cache c;
    int rc = check_cache(k, v, ks, vs, pt, B, false, &c);
    if (rc != TA_OK)
        return rc;
    const int64_t B_data = N > 0 ? B : 0;
    if ((rc = check_lens(counts, B)) != TA_OK || (starts && (rc = check_lens(starts, B)) != TA_OK))
        return rc;
    for (const ta_tensor *t : {ko, vo}) {
        rc = check_rows(t, ko->dtype, B, N, c.Hkv, c.D, true);
        if (rc != TA_OK && !(rc == TA_ERR_NULL && B_data == 0))     // (an output without rows needs no memory)
            return rc;
    }
    memset(r, 0, sizeof *r);
    r->kc = k->data; r->vc = v->data;
    r->ks = (const uint8_t *)ks->data; r->vs = (const uint8_t *)vs->data;
    r->k_out = ko->data; r->v_out = vo->data;
    r->page_table = pt ? (const int32_t *)pt->data : nullptr;
    r->starts = starts ? (const int32_t *)starts->data : nullptr;
    r->counts = (const int32_t *)counts->data;
    r->k_sp = k->stride[0]; r->k_sh = k->stride[1]; r->k_ss = k->stride[2];
    r->v_sp = v->stride[0]; r->v_sh = v->stride[1]; r->v_ss = v->stride[2];
    r->ks_sp = ks->stride[0]; r->ks_sh = ks->stride[1]; r->ks_ss = ks->stride[2];
    r->vs_sp = vs->stride[0]; r->vs_sh = vs->stride[1]; r->vs_ss = vs->stride[2];
    r->ko_sb = ko->stride[0]; r->ko_st = ko->stride[1]; r->ko_sh = ko->stride[2];
    r->vo_sb = vo->stride[0]; r->vo_st = vo->stride[1]; r->vo_sh = vo->stride[2];
    r->pt_sb = pt ? pt->stride[0] : 0;
    r->st_s = starts ? starts->stride[0] : 0;
    r->ct_s = counts->stride[0];
    r->B = (int)B; r->N = (int)N; r->Hkv = (int)c.Hkv; r->D = (int)c.D; r->ps = (int)c.ps;
    r->capacity = (int)c.capacity; r->n_pages = (int)c.n_pages;
    r->is_bf16 = ko->dtype == TA_BF16;
    r->vec = c.D % 16 == 0 && on_16_bytes(k) && on_16_bytes(v) && on_16_bytes(ko) && on_16_bytes(vo);
    r->tokens = tokens_per_group(B * N, 2 * c.Hkv, 32, 512);
    return TA_OK;
}

int ta_host_check_q8_compact(const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs, const ta_tensor *pt,
                             const ta_tensor *sl, const ta_tensor *ac, const ta_tensor *na, int32_t tree_size,
                             const ta_tensor *so, TAQ8Compact *c)
{
    if (!k || !v || !ks || !vs || !sl || !ac || !na)
        return TA_ERR_NULL;
    if (ac->ndim != 2)
        return TA_ERR_RANK;
    Cache cache;
    const int64_t B = ac->shape[0];
    if (B < 0 || B > TA_MAX_BATCH)
        return TA_ERR_BATCH;
    int rc = check_cache(k, v, ks, vs, pt, B, true, &cache);
    if (rc != TA_OK)
        return rc;
    // the rules of tree_attn_compact, whose element types this cache does not have
    ta_tensor kb = *k, vb = *v;
    kb.dtype = vb.dtype = TA_BF16;
    rc = ta_host_check_compact(&kb, &vb, pt, sl, ac, na, tree_size, so, c);
    if (rc != TA_OK)
        return rc;
    c->elem_bytes = 1;
    c->vec = cache.D % 16 == 0 && on_16_bytes(k) && on_16_bytes(v);
    c->ks = (uint8_t *)ks->data; c->vs = (uint8_t *)vs->data;
    c->ks_sp = ks->stride[0]; c->ks_sh = ks->stride[1]; c->ks_ss = ks->stride[2];
    c->vs_sp = vs->stride[0]; c->vs_sh = vs->stride[1]; c->vs_ss = vs->stride[2];
    return TA_OK;
}

int ta_host_build_q8_problem(const ta_tensor *q, const ta_tensor *k, const ta_tensor *v, const ta_tensor *ks, const ta_tensor *vs,
                             const ta_tensor *pt, const ta_tensor *sl, const ta_tensor *par, const ta_tensor *out,
                             const ta_tensor *lse, const ta_opts *opts, int num_cus, TAQ8Problem *qp)
{
    if (!q || !k || !v || !ks || !vs || !sl || !par || !out)
        return TA_ERR_NULL;
    if (k->dtype != TA_E4M3 || v->dtype != TA_E4M3 || ks->dtype != TA_E8M0 || vs->dtype != TA_E8M0)
        return TA_ERR_DTYPE;
    if (ks->ndim != 3 || vs->ndim != 3)
        return TA_ERR_RANK;
    const int kernel = opts ? opts->kernel : TA_KERNEL_AUTO;
    if (opts && (opts->k_new || opts->v_new || kernel < TA_KERNEL_AUTO || kernel > TA_KERNEL_MFMA_BASIC))
        return TA_ERR_OPTS;
    // the rules of tree_attn_fwd_ex hold for everything but the element types, which this cache does not share with q
    ta_tensor kq = *k, vq = *v;
    kq.dtype = vq.dtype = q->dtype;
    ta_opts o;
    memset(&o, 0, sizeof o);
    if (opts)
        o = *opts;
    o.kernel = TA_KERNEL_GENERIC;
    if (o.workspace && (uintptr_t)o.workspace % 256 != 0)
        return TA_ERR_WORKSPACE;
    o.workspace = nullptr;                                  // (looked at when the kernel is chosen)
    TAProblem &pr = qp->pr;
    if (pt && pt->ndim == 2 && pt->shape[1] > INT32_MAX)
        return TA_ERR_SHAPE;
    int rc = ta_host_build_problem(q, &kq, &vq, pt, sl, par, out, lse, &o, num_cus, &pr);
    if (rc != TA_OK)
        return rc;
    for (int i = 0; i < 3; ++i)
        if (ks->shape[i] != k->shape[i] || vs->shape[i] != k->shape[i])
            return TA_ERR_SHAPE;
    if (!strides_given(ks, false) || !strides_given(vs, false) || !no_zero_stride(out) || (lse && !no_zero_stride(lse)))
        return TA_ERR_STRIDE;
    if (pr.p.B > 0 && (!ks->data || !vs->data))
        return TA_ERR_NULL;
    if (pr.p.B > 0 && pr.p.n_pages < 1)
        return TA_ERR_SHAPE;
    pr.plan.table_row = -1;
    auto in_32_bits = [](const ta_tensor *t) { return t->stride[0] < INT32_MAX && t->stride[2] < INT32_MAX / 32; };    // (32 rows)
    const bool mfma_ok = (pr.p.D == 64 || pr.p.D == 128) && (!pt || pr.p.ps_shift >= 4) && pr.p.G <= 256 &&
                         on_16_bytes(q) && on_16_bytes(k) && on_16_bytes(v) && in_32_bits(k) && in_32_bits(v) && in_32_bits(ks) &&
                         in_32_bits(vs);
    if (!mfma_ok && (kernel == TA_KERNEL_MFMA || kernel == TA_KERNEL_MFMA_BASIC))
        return TA_ERR_OPTS;
    if (mfma_ok && kernel != TA_KERNEL_GENERIC) {
        rc = plan_mfma(out, opts, num_cus, &pr);
        if (rc != TA_OK)
            return rc;
    }
    if (opts && opts->workspace) {
        if (opts->workspace_bytes < pr.ws_bytes)
            return TA_ERR_WORKSPACE;
        pr.p.ws_o = (float *)opts->workspace;
        pr.p.ws_lse = (float *)((char *)opts->workspace + pr.ws_ls_off);
        pr.p.ws_parts = (int32_t *)((char *)opts->workspace + pr.ws_o_bytes + pr.ws_lse_bytes);
    }
    TAQ8Params &p = qp->p;
    memset(&p, 0, sizeof p);
    p.ks = (const uint8_t *)ks->data; p.vs = (const uint8_t *)vs->data;
    p.ks_sp = ks->stride[0]; p.ks_sh = ks->stride[1]; p.ks_ss = ks->stride[2];
    p.vs_sp = vs->stride[0]; p.vs_sh = vs->stride[1]; p.vs_ss = vs->stride[2];
    return TA_OK;
}

const TAQ8Params &ta_host_q8_params(TAQ8Problem *qp)
{
    static_cast<TAParams &>(qp->p) = qp->pr.p;
    qp->p.waves = qp->pr.plan.threads / TA_WAVE;
    return qp->p;
}

extern "C" {

int tree_attn_rope_freqs(const ta_rope_rule *rule, int32_t rotary_dim, float *freqs, float *amplitude)
{
    if (!rule || !freqs)
        return TA_ERR_NULL;
    if (rotary_dim < 2 || rotary_dim > TA_MAX_HEAD_DIM || rotary_dim % 2 != 0)
        return TA_ERR_HEAD_DIM;
    const bool bands = rule->rule == TA_ROPE_BANDS || rule->rule == TA_ROPE_YARN;
    if (rule->rule < TA_ROPE_PLAIN || rule->rule > TA_ROPE_YARN || rule->reserved != 0 || !(rule->base > 1.0) ||
        !isfinite(rule->base))
        return TA_ERR_OPTS;
    if (rule->rule != TA_ROPE_PLAIN && (!(rule->factor >= 1.0) || !isfinite(rule->factor)))
        return TA_ERR_OPTS;
    if (bands && (!(rule->original > 0.0) || !isfinite(rule->original) || !(rule->low >= 0.0) || !(rule->high > rule->low) ||
                  !isfinite(rule->high)))
        return TA_ERR_OPTS;
    for (int j = 0; j < rotary_dim / 2; ++j) {
        double f = pow(rule->base, -2.0 * j / rotary_dim);
        if (rule->rule == TA_ROPE_LINEAR) {
            f /= rule->factor;
        } else if (bands) {
            const double turns = rule->original * f / 6.283185307179586476925;
            double keep = (turns - rule->low) / (rule->high - rule->low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = keep * f + (1.0 - keep) * f / rule->factor;
        }
        freqs[j] = (float)f;
    }
    if (amplitude)
        *amplitude = rule->rule == TA_ROPE_YARN ? (float)(0.1 * log(rule->factor) + 1.0) : 1.f;
    return TA_OK;
}

int tree_attn_q8_plan(const ta_tensor *q, const ta_tensor *k_cache, const ta_tensor *v_cache, const ta_tensor *k_scale,
                      const ta_tensor *v_scale, const ta_tensor *page_table, const ta_tensor *seq_lens,
                      const ta_tensor *tree_parent, const ta_tensor *out, const ta_tensor *lse, const ta_opts *opts,
                      int32_t num_cus, int64_t plan[16])
{
    if (!plan)
        return TA_ERR_NULL;
    ta_opts o;
    if (opts) {
        o = *opts;
        o.workspace = nullptr;      // planning never needs the scratch itself
        o.workspace_bytes = 0;
    }
    TAQ8Problem qp;
    const int rc = ta_host_build_q8_problem(q, k_cache, v_cache, k_scale, v_scale, page_table, seq_lens, tree_parent, out, lse,
                                            opts ? &o : nullptr, num_cus > 0 ? num_cus : 256, &qp);
    if (rc != TA_OK)
        return rc;
    ta_host_fill_plan(qp.pr, plan);
    if (qp.pr.plan.kernel == TA_KERNEL_MFMA)
        plan[15] = qp.pr.plan.ks_rows;
    return TA_OK;
}

}  // extern "C"
