// Matrix-core KV pass over the 8-bit cache for gfx950: bf16 queries, head_dim 64 or 128, fp32 accumulation.
//
// For up to 32 query rows of a (request, KV head); more of them go to ta_q8_tile.hip.  As in the key-split kernel
// (ta_mfma_ks.hip) a workgroup keeps the rows and its waves split the
// KEYS of its share: wave w takes every NW-th run of 32 tokens with its own running softmax, moves its own codes HBM -> LDS into a
// ring that only it reads, and meets the others when the item ends.  What is different is the arithmetic, per 32 tokens:
//
//     S^T[token, row] = K . Q^T      v_mfma_f32_32x32x16_bf16: K's codes become bf16 values as they leave LDS (exact), and the
//                                    conversion takes the token's scale with it
//     O^T[d, row]    += V^T . P^T    V's codes are transposed out of LDS byte by byte and turned into bf16; P carries V's scales (powers
//                                    of two: the same rounding as without)
//
// Not taken: the 8-bit matrix instruction with the codes as they lie, K's scales as its own, and a query as the sum of two e4m3
// values.  It adds up products of neighbouring columns to 2^-13 of the largest only (measured with one large and one small product),
// and log-sum-exps of a few hundred tokens were off by up to 1.1e-4; these are off by less than 2e-6.
//
// The scales of a run, K's and V's, come with one load of a byte per lane ahead of V's codes.
//
// What bounds it: the loads.  128 requests of 8192 tokens, 8 KV heads, one new token with 4 heads each: 341 us with the merge, 6.3 TB/s,
// where a plain streaming read reaches 6.8; of 256 to 4096 tokens 103 us, 5.6 TB/s.  One request of 8192 tokens, one KV head: 14 us,
// two launches and the round trips of one share.
#include <initializer_list>
#include <type_traits>

#include "ta_q8.h"

typedef __bf16 q8_bf16x8 __attribute__((ext_vector_type(8)));
typedef float q8_f32x16 __attribute__((ext_vector_type(16)));
typedef int q8_i32x2 __attribute__((ext_vector_type(2)));

#define Q8_SUB 32                                // tokens a wave takes at a time
#define Q8_LENS 256                              // batches of up to this many requests keep their lengths in LDS

__device__ __forceinline__ float q8_swap_max(float x)      // over the two lanes that share a query row
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ uint32_t q8_quad_max(uint32_t x)            // over four neighbouring lanes
{
    auto up = [&](uint32_t y) { x = y > x ? y : x; };
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));     // lanes 1 0 3 2 of every four
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));     // 2 3 0 1
    return x;
}

__device__ __forceinline__ uint32_t q8_row16_max(uint32_t x)           // over sixteen neighbouring lanes
{
    x = q8_quad_max(x);
    auto up = [&](uint32_t y) { x = y > x ? y : x; };
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));    // mirrored within eight
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));    // rotated by eight within sixteen
    return x;
}

// Eight codes times a power of two as bf16.
__device__ __forceinline__ uint4 q8_bf16_8(int lo, int hi, float scale)
{
    return make_uint4(q8_bf16_2<false>((uint32_t)lo, scale), q8_bf16_2<true>((uint32_t)lo, scale),
                      q8_bf16_2<false>((uint32_t)hi, scale), q8_bf16_2<true>((uint32_t)hi, scale));
}

__device__ __forceinline__ void q8_lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int N>
__device__ __forceinline__ void q8_vm_wait()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Every lane moves 16 bytes from its global address to LDS lds_wave_base + 16 * lane (or a byte to a word of its own, 4 * lane).
// (nt: nobody else reads what is loaded, and a stream that is read once passes by faster: one new token of 128 requests 116 us,
// 122 without.)
#define Q8_DMA(text, ...) asm volatile("s_mov_b32 m0, %[m]\n\ts_nop 0\n\t" text ::__VA_ARGS__ : "memory")

__device__ __forceinline__ void q8_dma(const void *gptr, uint32_t lds_wave_base)
{
    Q8_DMA("global_load_lds_dwordx4 %[a], off nt", [a] "v"(gptr), [m] "s"(lds_wave_base));
}

__device__ __forceinline__ void q8_dma_byte(const void *gptr, uint32_t lds_wave_base)
{
    Q8_DMA("global_load_lds_ubyte %[a], off nt", [a] "v"(gptr), [m] "s"(lds_wave_base));
}

__device__ __forceinline__ void q8_dma_s(const void *base, uint32_t off, uint32_t lds_wave_base)
{
    Q8_DMA("global_load_lds_dwordx4 %[o], %[b] nt", [o] "v"(off), [b] "s"(base), [m] "s"(lds_wave_base));
}

// Two or four such loads in a row, 1 KB apart in memory and in LDS (the instruction's offset counts on both sides).
__device__ __forceinline__ void q8_dma_2k(const void *base, uint32_t o0, uint32_t o1, uint32_t lds_wave_base)
{
    Q8_DMA("global_load_lds_dwordx4 %[o], %[b] nt\n\tglobal_load_lds_dwordx4 %[p], %[b] offset:0x400 nt",
           [o] "v"(o0), [p] "v"(o1), [b] "s"(base), [m] "s"(lds_wave_base));
}

__device__ __forceinline__ void q8_dma_4k(const void *base, uint32_t o0, uint32_t o1, uint32_t lds_wave_base)
{
    Q8_DMA("global_load_lds_dwordx4 %[o], %[b] nt\n\tglobal_load_lds_dwordx4 %[p], %[b] offset:0x400 nt\n\t"
           "global_load_lds_dwordx4 %[o], %[b] offset:0x800 nt\n\tglobal_load_lds_dwordx4 %[p], %[b] offset:0xc00 nt",
           [o] "v"(o0), [p] "v"(o1), [b] "s"(base), [m] "s"(lds_wave_base));
}

// Sizes of one instance.  NW: waves of a workgroup; OCC: workgroups per compute unit, which share
// its LDS.  A wave's ring holds NS runs of 32 tokens of K and as many of V; at the end it stages a block's fp32 results there.
template <int DH, int NW, int OCC>
struct Q8Shape {
    static constexpr int ROW = DH;                         // bytes of a token row
    static constexpr int SUBB = Q8_SUB * ROW;              // bytes of 32 K (or V) rows
    static constexpr int REGION = 128 * 1024 / OCC / NW;   // LDS of a wave
    static constexpr int RING = NW * REGION;
    static constexpr int NS = REGION / (2 * SUBB);         // runs in flight
    static constexpr int LD = SUBB / 1024;                 // 1 KB loads per run of K (or V)
    static constexpr int RPL = Q8_SUB / LD;                // token rows per load
    static constexpr int ROWS = 32;
    static constexpr int NT = 64 * NW;
    static constexpr int QB = ROWS * 2 * DH;               // bytes of the Q rows
    static constexpr int QP = (ROWS * DH / 8 + NT - 1) / NT;      // 16-byte pieces of bf16 rows a thread loads
    static constexpr int FIXED = RING + QB + 4 * NW * NS * 64 + 4 * 2 * NW * ROWS + 4 * NW;
    static_assert(NS >= 2 && NS <= 4 && REGION >= 32 * DH * 4, "ring and staging area");
    static_assert(NW >= 4 && NW % 4 == 0, "at most one of a list's last three runs per wave; results are added up in fours");
};

// What a workgroup's lists are.  Q8_CUT: a share of the line of all lists.  Q8_SOLO: workgroup x walks list x from end to end (see
// p.solo).
enum { Q8_CUT, Q8_SOLO };

template <int DH, int NW, int OCC, int MODE>
static constexpr size_t q8_smem(int B)
{
    return Q8Shape<DH, NW, OCC>::FIXED + (MODE == Q8_SOLO || B <= TA_WAVE ? 0 : sizeof(int) * (B + 2 + (B <= Q8_LENS ? 2 * B : 0)));
}

template <int DH, int NW, int OCC, int MODE>
__global__ __launch_bounds__(64 * NW, OCC * NW / 4) void ta_q8_kv_kernel(TA_SCHED_PARAMS, TAQ8Params p)
{
    const TASched sc = TA_SCHED;
    using C = Q8Shape<DH, NW, OCC>;
    constexpr bool SOLO = MODE == Q8_SOLO;
    constexpr int NKK = DH / 16, NDB = DH / 32, SLOTS = DH / 16, QSLOTS = DH / 8;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    char *const qrows = smem + C::RING;                                 // Q rows of the item
    uint32_t *const scales = (uint32_t *)(qrows + C::QB);                // [NW][NS][64]: a run's scales, K's, then V's
    float *const stat = (float *)(scales + NW * C::NS * 64);             // [NW][2][ROWS]: reference and sum
    int *const wbad = (int *)(stat + 2 * NW * C::ROWS);                  // [NW]: TA_STATUS_* bits a wave has met
    int *const cum = wbad + NW;                                          // more than 64 requests: [B + 1] schedule
    int *const lens = cum + sc.B + 1, *const starts = lens + sc.B;       // and, up to Q8_LENS, lengths and window starts
    const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) char *)smem);

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, hf = lane >> 5;
    // Schedule (see ta_build_schedule).  Up to 64 requests every wave keeps it in registers, lane b for request b: no
    // exchange between the waves, which start on their own.
    const bool in_regs = sc.B <= TA_WAVE;
    int s_len = 0, s_start = 0, s_units = 0, s_cum = 0, total;
    int t, t_end;
    if constexpr (SOLO) {
        s_len = sc.seq_lens[(int64_t)(w / sc.Hkv) * sc.sl_s];
        s_start = ta_kv_start(sc, w / sc.Hkv);
        ta_touch_args<TAParams>(s_len);
        t = 0;
        t_end = 1;
    } else {
        if (in_regs) {
            if (lane < sc.B) {
                s_len = sc.seq_lens[(int64_t)lane * sc.sl_s];
                s_start = ta_kv_start(sc, lane);
            }
            ta_touch_args<TAParams>();
            if (lane < sc.B)
                s_units = ta_list_tiles(sc, s_len, s_start) + sc.pad;
            s_cum = ta_wave_scan(s_units);
            total = sc.Hkv * __builtin_amdgcn_readlane(s_cum, 63);
        } else {
            total = sc.Hkv * ta_build_schedule(sc, cum, sc.B <= Q8_LENS ? lens : nullptr, sc.B <= Q8_LENS ? starts : nullptr);
        }
        ta_wg_range(sc, total, w, t, t_end);
        t = __builtin_amdgcn_readfirstlane(t);
        t_end = __builtin_amdgcn_readfirstlane(t_end);
    }
    const float c = p.scale_log2e;
    const bool paged = p.page_table != nullptr;
    const uint32_t ksp = (uint32_t)p.k_sp, kss = (uint32_t)p.k_ss, vsp = (uint32_t)p.v_sp, vss = (uint32_t)p.v_ss;
    // 16-byte slots of a row in LDS: K slot s of row r holds chunk s ^ kx(r), V slot s chunk s ^ 2 vx(r); both spread the rows that
    // a fragment read touches at once over all banks
    auto kx = [](int r) { return DH == 64 ? (r >> 2) & 3 : (r >> 1) & 7; };
    auto qx = [](int r) { return DH == 64 ? (r >> 1) & 7 : r & 15; };      // (the same for rows of Q, and their bf16 slots)
    auto vx = [](int r) { return DH == 64 ? (r >> 3) & 1 : ((r >> 1) & 1) | (((r >> 3) & 1) << 1); };
    const uint32_t region = lds0 + wave * C::REGION;
    char *const kring = smem + wave * C::REGION, *const vring = kring + C::NS * C::SUBB;
    uint32_t *const sring = scales + wave * C::NS * 64;
    const uint32_t sregion = lds0 + (uint32_t)((char *)sring - smem);
    // fragment offsets of this lane inside a run
    const int kf_row = r32 * C::ROW, kf_x = kx(r32);
    const int vrho = (lane >> 1) & 7, vtk = 4 * hf + (vrho & 3) + 8 * (vrho >> 2), vh16 = (lane >> 4) & 1;
    const int vf_row = vtk * C::ROW + (lane & 1) * 8, vf_x = 2 * vx(vtk);
    // load role of this lane: row lrow of the RPL rows of a load, slot dslot
    const int lrow = lane / SLOTS, dslot = lane % SLOTS;
    constexpr int OFFS = DH == 64 ? 1 : 2;                                 // the placement repeats after that many loads
    uint32_t koff[OFFS], voff[OFFS];                                       // lane offset from the load's first row
#pragma unroll
    for (int k = 0; k < OFFS; ++k) {
        koff[k] = lrow * kss + (dslot ^ kx(k * C::RPL + lrow)) * 16;
        voff[k] = lrow * vss + (dslot ^ (2 * vx(k * C::RPL + lrow))) * 16;
    }
    // whole runs: 32 rows one after the other in memory
    const bool dense = (!paged || p.ps_shift >= 5) && kss == DH && vss == DH;
    // page ids a wave keeps: lane l holds the page of part l % ppr of its run pg_base + l / ppr
    const int ppr_shift = !paged || p.ps_shift >= 5 ? 0 : 1;               // log2 of pages per run (pages hold 16 tokens or more)
    // scales: lanes below 32 load those of K, the others those of V
    const uint32_t ssp = (uint32_t)(hf ? p.vs_sp : p.ks_sp), sss = (uint32_t)(hf ? p.vs_ss : p.ks_ss);
    // what an item's start and end derive from the thread id is derived there: hoisted, it would be spilled in the loop
    auto fresh_lane = [&]() {
        int x = lane;
        asm volatile("" : "+v"(x));
        return x;
    };

    // ---- the current item: a list (b, g), its tiles [j0, j1), i.e. the prefix tokens [max(lo, S), hi), walked in runs of
    // 32 from lo, and the T tree tokens; run u belongs to wave u % NW
    int b = -1, g = 0, slot = 0, L = 0, S = 0, lo = 0, hi = 0, n_pre = 0, n_sub = 0, n_full = 0, bad = 0;
    bool has_tree = false;
    uint4 q_piece[C::QP] = {};                             // this thread's pieces of the item's Q rows
    int pg = 0, pg_first = 0, pg_last = 0, parent = 0;     // pages of full runs, of the first and of the last run; tree
    unsigned long long gmask = 0;
    const uint8_t *kgp = nullptr, *vgp = nullptr, *sgp = nullptr;
    auto sub_pos = [&](int u) { return u < n_pre ? lo + u * Q8_SUB : L + (u - n_pre) * Q8_SUB; };
    auto sub_end = [&](int u) { return u < n_pre ? min(hi, lo + (u + 1) * Q8_SUB) : L + min(sc.T, (u - n_pre + 1) * Q8_SUB); };
    // this wave's run among those that are not full: the ragged end of the prefix and the tree's (n_sub: none)
    auto last_own = [&]() {
        const int u = n_full + ((wave - n_full) & (NW - 1));
        return u < n_sub ? u : n_sub;
    };
    auto page_of = [&](int pos) { return p.page_table[(int64_t)b * p.pt_sb + (pos >> p.ps_shift)]; };
    auto load_pages = [&](int i0) {                        // pages of this wave's full runs i0, i0 + 1, ...
        const int l = fresh_lane();
        const int pos = lo + (wave + NW * (i0 + (l >> ppr_shift))) * Q8_SUB + (l & ((1 << ppr_shift) - 1)) * (Q8_SUB >> ppr_shift);
        return pos >= S && pos < lo + n_full * Q8_SUB ? page_of(pos) : 0;
    };
    // Moves on to the next item of [t, t_end) and requests what its start needs: Q, page ids, parents.  False at the end.
    auto next_item = [&]() {
        while (t < t_end) {
            int n_b, j0, j1;
            if constexpr (SOLO) {
                t = t_end;
                b = w / sc.Hkv;
                g = w - b * sc.Hkv;
                L = s_len;
                S = s_start;
                n_b = ta_list_tiles(sc, L, S);
                j0 = 0;
                j1 = n_b;
            } else {
                int cum_b, cum_e;
                if (in_regs) {
                    b = __popcll(__ballot(sc.Hkv * s_cum <= t));
                    cum_e = __builtin_amdgcn_readlane(s_cum, b);
                    cum_b = cum_e - __builtin_amdgcn_readlane(s_units, b);
                } else {
                    if (b < 0)
                        b = ta_find_request(sc, cum, t);
                    else if ((int64_t)sc.Hkv * cum[b + 1] <= t)
                        ++b;
                    b = __builtin_amdgcn_readfirstlane(b);
                    cum_b = __builtin_amdgcn_readfirstlane(cum[b]);
                    cum_e = __builtin_amdgcn_readfirstlane(cum[b + 1]);
                }
                const int n_u = cum_e - cum_b;                          // schedule units of one list
                g = (t - sc.Hkv * cum_b) / n_u;
                const int seg_start = sc.Hkv * cum_b + g * n_u;
                n_b = n_u - sc.pad;
                j0 = t - seg_start;
                j1 = min(n_b, t_end - seg_start);
                if (j1 <= j0) {
                    t = seg_start + n_u;                               // t lies in the list's trailing padding
                    continue;
                }
                t = seg_start + (j1 == n_b ? n_u : j1);
                slot = w + b * sc.Hkv + g;
                ta_note_owner(p, b, g, w, j0, j1, n_b);
                if (in_regs) {
                    L = __builtin_amdgcn_readlane(s_len, b);
                    S = __builtin_amdgcn_readlane(s_start, b);
                } else {
                    L = __builtin_amdgcn_readfirstlane(sc.B <= Q8_LENS ? lens[b] : sc.seq_lens[(int64_t)b * sc.sl_s]);
                    S = __builtin_amdgcn_readfirstlane(sc.B <= Q8_LENS ? starts[b] : ta_kv_start(sc, b));
                }
            }
            bad = ta_request_ok(sc, L, S) ? 0 : TA_STATUS_BAD_SEQLEN;
            const int tile0 = bad ? 0 : S / TA_TILE;
            has_tree = j1 == n_b;
            const int jp = has_tree ? n_b - 1 : j1;
            lo = max((tile0 + j0) * TA_TILE, S) & ~(Q8_SUB - 1);
            hi = min((tile0 + jp) * TA_TILE, L);
            n_pre = !bad && hi > lo ? (hi - lo + Q8_SUB - 1) / Q8_SUB : 0;
            n_full = !bad && hi > lo ? (hi - lo) / Q8_SUB : 0;
            n_sub = bad ? 0 : n_pre + (has_tree ? (sc.T + Q8_SUB - 1) / Q8_SUB : 0);
            kgp = (const uint8_t *)p.k + (int64_t)g * p.k_sh;
            vgp = (const uint8_t *)p.v + (int64_t)g * p.v_sh;
            sgp = hf ? p.vs + (int64_t)g * p.vs_sh : p.ks + (int64_t)g * p.ks_sh;
            const int l = fresh_lane();
#pragma unroll
            for (int i = 0; i < C::QP; ++i) {
                // rows past the group's end repeat its first row (their results are never stored)
                const int x = i * C::NT + wave * 64 + l, row = x / QSLOTS;
                if (C::ROWS * QSLOTS >= C::NT || row < C::ROWS) {
                    const int R = row < p.rows ? row : 0;
                    const int node = (int)__umulhi((uint32_t)R << 8, p.g_magic);      // R / G
                    q_piece[i] = *(const uint4 *)((const uint16_t *)p.q + (int64_t)b * p.q_sb + (int64_t)node * p.q_st +
                                               (int64_t)(g * p.G + R - node * p.G) * p.q_sh + 8 * (x % QSLOTS));
                }
            }
            if (wave >= n_sub)
                return true;                                       // nothing to walk for this wave
            const int ul = last_own();
            if (paged) {
                pg = load_pages(0);
                // runs that are not full: lane r holds the page of row r
                if (wave == 0)
                    pg_first = page_of(max(lo, S) + min(l & 31, sub_end(0) - 1 - max(lo, S)));
                if (ul < n_sub)
                    pg_last = page_of(max(S, min(sub_pos(ul) + (l & 31), sub_end(ul) - 1)));
            }
            if (ul < n_sub && ul >= n_pre && l < sc.T) {
                if (p.masks_in)
                    gmask = ta_given_mask(p, b, l);
                else
                    parent = p.parent[(int64_t)b * p.par_sb + l];
            }
            return true;
        }
        return false;
    };
    auto checked = [&](int id) {                           // a page id as an address: one outside the cache is reported
        if (!ta_page_ok(p, id)) {
            bad |= TA_STATUS_BAD_PAGE;
            id = 0;
        }
        return id;
    };

    bool more = next_item();
    while (more) {
        q8_f32x16 o[NDB];
        float m_run, l_run;
        unsigned long long tmask;
        m_run = -INFINITY;
        l_run = 0.f;
        tmask = ~0ull;
        const int u_last = last_own();
        int u = wave, pg_base = 0;
        // everything requested is here: no wait of the compiler for it may fall behind the loads into LDS, which it does
        // not know of
#pragma unroll
        for (int i = 0; i < C::QP; ++i)
            asm volatile("" : "+v"(q_piece[i].x), "+v"(q_piece[i].y), "+v"(q_piece[i].z), "+v"(q_piece[i].w));
        if (u < n_sub) {
            asm volatile("" : "+v"(pg), "+v"(pg_first), "+v"(pg_last), "+v"(parent), "+v"(gmask));
            if (paged) {
                pg = checked(pg);
                pg_first = checked(pg_first);
                pg_last = checked(pg_last);
            }
        }

        // Loads of run u into ring slot sl: K part, LD loads of 1 KB, or V part, one load of both scales and LD of 1 KB.
        auto issue = [&](int u, int sl, bool is_v) {
            const uint32_t dst = region + (is_v ? C::NS * C::SUBB : 0) + sl * C::SUBB;
            const uint32_t sdst = sregion + sl * 256;
            const uint32_t sp = is_v ? vsp : ksp, ss = is_v ? vss : kss;
            const uint8_t *gp = is_v ? vgp : kgp;
            const int pos0 = sub_pos(u);
            const bool full = u < n_full && pos0 >= S;
            if (full) {
                const int pl = ((u - wave) / NW - pg_base) << ppr_shift;           // lane that holds the run's first page
                const uint32_t page0 = paged ? (uint32_t)__builtin_amdgcn_readlane(pg, pl) : (uint32_t)b;
                const uint32_t page1 = ppr_shift ? (uint32_t)__builtin_amdgcn_readlane(pg, pl + 1) : page0;
                const uint32_t sr0 = paged ? (uint32_t)(pos0 & (p.ps - 1)) : (uint32_t)pos0;
                if (is_v) {
                    const uint32_t page = r32 < 16 ? page0 : page1;
                    const uint32_t sr = ppr_shift ? (uint32_t)(r32 & 15) : sr0 + (uint32_t)r32;
                    q8_dma_byte(sgp + (uint64_t)page * ssp + (uint64_t)sr * sss, sdst);
                }
                if (dense) {
                    const char *base = (const char *)(gp + (uint64_t)page0 * sp + (uint64_t)sr0 * DH);
                    if constexpr (DH == 128)
                        q8_dma_4k(base, is_v ? voff[0] : koff[0], is_v ? voff[OFFS - 1] : koff[OFFS - 1], dst);
                    else
                        q8_dma_2k(base, is_v ? voff[0] : koff[0], is_v ? voff[0] : koff[0], dst);
                } else {
#pragma unroll
                    for (int k = 0; k < C::LD; ++k) {
                        const int r0 = k * C::RPL;
                        const uint32_t page = r0 < 16 ? page0 : page1;
                        const uint32_t sr = ppr_shift ? (uint32_t)(r0 & 15) : sr0 + (uint32_t)r0;
                        q8_dma_s(gp + (uint64_t)page * sp + (uint64_t)sr * ss, is_v ? voff[k % OFFS] : koff[k % OFFS], dst + k * 1024);
                    }
                }
            } else {
                // rows past the run's end and rows before the window start read an attended token of the run (their
                // probabilities are exactly zero)
                const int first = max(pos0, S), end = sub_end(u);
                const int pgr = u == u_last ? pg_last : pg_first;
                // (the first run's pages are kept from its first attended row on)
                auto place = [&](int row, uint32_t &page, uint32_t &sr) {
                    int pos = pos0 + row;
                    pos = pos < end && pos >= first ? pos : first;
                    page = paged ? (uint32_t)__shfl(pgr, pos - (u == u_last ? pos0 : first), TA_WAVE) : (uint32_t)b;
                    sr = paged ? (uint32_t)(pos & (p.ps - 1)) : (uint32_t)pos;
                };
                uint32_t page, sr;
                if (is_v) {
                    place(r32, page, sr);
                    q8_dma_byte(sgp + (uint64_t)page * ssp + (uint64_t)sr * sss, sdst);
                }
#pragma unroll
                for (int k = 0; k < C::LD; ++k) {
                    const int row = k * C::RPL + lrow;
                    place(row, page, sr);
                    const int chunk = dslot ^ (is_v ? 2 * vx(row) : kx(row));
                    q8_dma(gp + (uint64_t)page * sp + (uint64_t)sr * ss + chunk * 16, dst + k * 1024);
                }
            }
        };
#pragma unroll 1
        for (int k = 0; k < 2 * C::NS; ++k)                    // K and V of the wave's first runs
            if (u + (k >> 1) * NW < n_sub)
                issue(u + (k >> 1) * NW, k >> 1, k & 1);

        {
            const int l = fresh_lane();
#pragma unroll
            for (int i = 0; i < C::QP; ++i) {
                const int x = i * C::NT + wave * 64 + l, row = x / QSLOTS;
                if (C::ROWS * QSLOTS >= C::NT || row < C::ROWS)
                    *(uint4 *)(qrows + row * 2 * DH + (((x % QSLOTS) ^ qx(row)) << 4)) = q_piece[i];
            }
        }
        q8_lds_barrier();
        // while the first runs are on their way: Q fragments into every wave's registers (one block of rows), O = 0 and, in a wave
        // that has tree tokens, the ancestor masks
        // (a lane's sixteen codes of a chunk are columns 32 j + 16 hf .. + 15: two products' worth, and Q's pieces go with them)
        auto q_frag = [&](int kk) {
            return *(const uint4 *)(qrows + r32 * 2 * DH + (((4 * (kk >> 1) + 2 * hf + (kk & 1)) ^ qx(r32)) << 4));
        };
        uint4 qf[NKK];
        if (u < n_sub) {
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk)
                qf[kk] = q_frag(kk);
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[db][i] = 0.f;
        if (u_last < n_sub && u_last >= n_pre) {
            // lane i walks up from node i
            const int l = fresh_lane();
            unsigned long long m = 0;
            bool wrong = false;
            if (p.masks_in) {
                m = gmask;
                wrong = l < sc.T && !ta_given_mask_ok(m, l);
            } else {
                int cur = l < sc.T ? l : -1;
                for (int steps = 0; __any(cur >= 0); ++steps) {
                    wrong |= cur >= 0 && (cur >= sc.T || steps >= sc.T);
                    if (cur >= 0)
                        m |= 1ull << (cur & 63);
                    const int up = __shfl(parent, cur & 63, TA_WAVE);
                    cur = cur >= 0 && !wrong ? up : -1;
                }
            }
            if (__any(wrong))
                bad |= TA_STATUS_BAD_PARENT;
            const int row = (l & 31);
            const int node = p.q_off + (int)__umulhi((uint32_t)row << 8, p.g_magic);
            const uint32_t m_lo = __shfl((uint32_t)m, node & 63, TA_WAVE), m_hi = __shfl((uint32_t)(m >> 32), node & 63, TA_WAVE);
            if (row < p.rows)
                tmask = ((unsigned long long)m_hi << 32) | m_lo;
        }

        int sl = 0;
#pragma unroll 1
        for (; u < n_sub; u += NW) {
            const int un = u + C::NS * NW;
            const int left = (n_sub - 1 - u) / NW, later = min(left, C::NS - 1);   // runs of this wave behind this one; requested
            const bool ahead = un < n_sub;
            constexpr int RUN = 2 * C::LD + 1;                                     // loads of a run
            if (later >= 3)
                q8_vm_wait<C::LD + 3 * RUN>();
            else if (later == 2)
                q8_vm_wait<C::LD + 2 * RUN>();
            else if (later == 1)
                q8_vm_wait<C::LD + RUN>();
            else
                q8_vm_wait<C::LD>();
            // ---- scales: a lane of the upper half turns the byte of its token into V's factor
            uint32_t *const ssl = sring + sl * 64;
            const int pos0 = sub_pos(u), cnt = sub_end(u) - pos0;
            const bool tree = u >= n_pre;
            const uint32_t own = ssl[32 + r32];
            const float ks = q8_scale(ssl[r32]);
            if (hf)
                ssl[32 + r32] = __float_as_uint(q8_scale(own));
            // ---- S^T = K . Q^T
            q8_f32x16 s;
            const char *kt = kring + sl * C::SUBB + kf_row;
#pragma unroll
            for (int j = 0; j < NKK / 2; ++j) {
                const uint4 x = *(const uint4 *)(kt + (((2 * j + hf) ^ kf_x) << 4));
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const int kk = 2 * j + k2;
                    const uint4 kf = q8_bf16_8(k2 ? x.z : x.x, k2 ? x.w : x.y, ks);
                    const q8_f32x16 z = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(q8_bf16x8, kf), __builtin_bit_cast(q8_bf16x8, qf[kk]),
                                                                kk == 0 ? z : s, 0, 0, 0);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // the K rows are in registers: their slot is free
            if (ahead) {
                const int i = (un - wave) / NW - pg_base;
                if (paged && (i << ppr_shift) >= TA_WAVE) {
                    pg_base += i;                                          // the next page ids (waits for all loads)
                    pg = checked(load_pages(pg_base));
                }
                issue(un, sl, false);
            }
            // ---- scores of tokens that do not exist, or that are no ancestors, become -inf
            uint32_t seen;
            const bool masked = tree || cnt < Q8_SUB || pos0 < S;
            if (masked) {
                uint32_t vm = cnt < Q8_SUB ? (1u << cnt) - 1u : ~0u;
                if (!tree && pos0 < S)
                    vm &= ~((1u << (S - pos0)) - 1u);
                uint32_t mm = vm;
                if (tree)
                    mm &= (uint32_t)(tmask >> ((u - n_pre) * Q8_SUB));
                seen = mm;
                mm >>= 4 * hf;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((mm >> (8 * (i / 4) + (i % 4))) & 1u))
                        s[i] = -INFINITY;
            }
            // ---- running softmax
            float t0 = s[0], t1 = s[1], t2 = s[2], t3 = s[3];
#pragma unroll
            for (int i = 4; i < 16; i += 4) {
                t0 = fmaxf(t0, s[i]);
                t1 = fmaxf(t1, s[i + 1]);
                t2 = fmaxf(t2, s[i + 2]);
                t3 = fmaxf(t3, s[i + 3]);
            }
            const float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * c;           // of this lane's sixteen scores
            // (the reference moves only when a score exceeds it by more than 2^4: see ta_mfma_ks.hip)
            if (__any(top > m_run + (SOLO ? 0.f : 4.f))) {
                const float m_new = fmaxf(m_run, q8_swap_max(top));
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[db][i] *= alpha;
            }
            // ---- V.  Younger than it: the runs behind, and the K part just requested
            if (ahead)
                q8_vm_wait<(C::NS - 1) * RUN + C::LD>();
            else if (later >= 3)
                q8_vm_wait<3 * RUN>();
            else if (later == 2)
                q8_vm_wait<2 * RUN>();
            else if (later == 1)
                q8_vm_wait<RUN>();
            else
                q8_vm_wait<0>();
            char *const vt = vring + sl * C::SUBB;
            if (tree) {
                // A NaN of a node counts only for rows that attend to it: it is taken out of the product, where zero times it would
                // spoil them all, and their outputs are made NaN.  (In the prefix every row attends to every token.)
                uint32_t any = q8_scale(own) != q8_scale(own) ? 0x80u : 0u;
                uint4 *const half = (uint4 *)(vt + r32 * C::ROW + hf * (C::ROW / 2));
                auto nans = [](uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };      // 0x80 in each byte that is one
#pragma unroll
                for (int k = 0; k < SLOTS / 2; ++k) {
                    const uint4 x = half[k];
                    any |= nans(x.x) | nans(x.y) | nans(x.z) | nans(x.w);
                }
                const unsigned long long hit = __ballot(any != 0);
                if (hit) {
                    auto clear = [&](uint32_t x) { const uint32_t n = nans(x) >> 7; return x & ~(n * 0xffu); };
#pragma unroll 1
                    for (int k = 0; k < SLOTS / 2; ++k) {
                        const uint4 x = half[k];
                        half[k] = make_uint4(clear(x.x), clear(x.y), clear(x.z), clear(x.w));
                    }
                    const uint32_t tokens = (uint32_t)hit | (uint32_t)(hit >> 32);
                    if (hf && q8_scale(own) != q8_scale(own))
                        ssl[32 + r32] = 0u;
                    if (seen & tokens) {
#pragma unroll
                        for (int db = 0; db < NDB; ++db)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                o[db][i] = __uint_as_float(0x7fc00000u);
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            }
            // All fragments are requested here and arrive under the exponentials
            typedef __attribute__((address_space(3))) q8_i32x2 *lds_i2;
            q8_i32x2 vf[2][NDB];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int db = 0; db < NDB; ++db)
                    vf[kb][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (lds_i2)(vt + vf_row + kb * 16 * C::ROW + (((2 * db + vh16) ^ vf_x) << 4)));
            __builtin_amdgcn_sched_barrier(0);
            uint4 pb[2];
            // (a row that has not seen a token yet keeps -inf: its probabilities are exp2(-inf) = 0)
            const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
            float sum = 0.f;
            uint32_t pk[8];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const uint4 vs = *(const uint4 *)(ssl + 32 + 8 * i4 + 4 * hf);       // V's factors of the lane's four tokens
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e[i] = __builtin_amdgcn_exp2f(fmaf(s[4 * i4 + i], c, neg_m));
                sum += (e[0] + e[1]) + (e[2] + e[3]);
                pk[2 * i4] = q8_pack_bf16(e[0] * __uint_as_float(vs.x), e[1] * __uint_as_float(vs.y));
                pk[2 * i4 + 1] = q8_pack_bf16(e[2] * __uint_as_float(vs.z), e[3] * __uint_as_float(vs.w));
            }
            l_run += sum;
            pb[0] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            pb[1] = make_uint4(pk[4], pk[5], pk[6], pk[7]);
            // ---- O^T += V^T . P^T
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int db = 0; db < NDB; ++db) {
                    const uint4 a = q8_bf16_8(vf[kb][db].x, vf[kb][db].y, 1.f);
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(q8_bf16x8, a),
                                                                        __builtin_bit_cast(q8_bf16x8, pb[kb]),
                                                                        o[db], 0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // the V rows are in registers
            if (ahead)
                issue(un, sl, true);
            sl = sl + 1 < C::NS ? sl + 1 : 0;
        }

        // ---- the waves' results meet, a block of rows at a time: each stages its 32 x DH block (16-byte chunk ch of row r at chunk
        // ch ^ (r & 15)) in its own part of the ring, then every thread adds up its columns of one row over the waves
        const int n_live = min(NW, (n_sub + 3) & ~3);          // waves that had runs, in fours
        const int l_e = fresh_lane(), r32_e = l_e & 31, hf_e = l_e >> 5;
        {
            int wb = 0;
            if (__any(bad)) {
                for (int bit : {TA_STATUS_BAD_PARENT, TA_STATUS_BAD_SEQLEN, TA_STATUS_BAD_PAGE})
                    wb |= __any(bad & bit) ? bit : 0;
            }
            if (l_e == 0)
                wbad[wave] = wb;
            const float l_tot = l_run + __shfl_xor(l_run, 32, TA_WAVE);
            if (hf_e == 0) {
                stat[(wave * 2 + 0) * C::ROWS + r32_e] = m_run;
                stat[(wave * 2 + 1) * C::ROWS + r32_e] = l_tot;
            }
        }
        const int slot_e = slot, b_e = b, g_e = g;
        if (wave < n_live) {                               // (nobody reads what the others would put there)
            float *stage = (float *)(smem + wave * C::REGION);
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const int ch = db * 8 + 2 * i4 + hf_e;
                    *(float4 *)(stage + r32_e * DH + ((ch ^ (r32_e & 15)) << 2)) =
                        make_float4(o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]);
                }
        }
        more = next_item();                                // its requests are on their way during the rest
        q8_lds_barrier();
        int any_bad = 0;
#pragma unroll
        for (int k = 0; k < NW; ++k)
            any_bad |= wbad[k];
        const int x_e = wave * 64 + l_e;
        constexpr int TPR = 16, CPT = DH / TPR;            // threads per row, columns per thread
#pragma unroll 1
        for (int row = x_e / TPR; row < 32; row += C::NT / TPR) {
            const int c0 = (x_e % TPR) * (CPT / 4);
            float mw[NW], big = -INFINITY;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                mw[k] = stat[(k * 2 + 0) * C::ROWS + row];
                big = fmaxf(big, mw[k]);
            }
            float l_tot = 0.f, acc[CPT];
#pragma unroll
            for (int i = 0; i < CPT; ++i)
                acc[i] = 0.f;
#pragma unroll
            for (int k0 = 0; k0 < NW; k0 += 4)
                if (k0 < n_live) {
#pragma unroll
                    for (int k = k0; k < k0 + 4; ++k) {
                        const float wgt = mw[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[k] - big);
                        l_tot = fmaf(wgt, stat[(k * 2 + 1) * C::ROWS + row], l_tot);
#pragma unroll
                        for (int q = 0; q < CPT / 4; ++q) {
                            const float4 x = *(const float4 *)(smem + k * C::REGION + (row * DH + (((c0 + q) ^ (row & 15)) << 2)) * 4);
                            acc[4 * q + 0] = fmaf(wgt, x.x, acc[4 * q + 0]);
                            acc[4 * q + 1] = fmaf(wgt, x.y, acc[4 * q + 1]);
                            acc[4 * q + 2] = fmaf(wgt, x.z, acc[4 * q + 2]);
                            acc[4 * q + 3] = fmaf(wgt, x.w, acc[4 * q + 3]);
                        }
                    }
                }
            const float inv = any_bad ? 0.f : 1.f / l_tot;
            // largest magnitude of the row, as bits: those of a NaN are above all others
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < CPT; ++i) {
                acc[i] *= inv;
                top = max(top, __float_as_uint(acc[i]) & 0x7fffffffu);
            }
            top = q8_row16_max(top);
            const bool nan_seen = top > 0x7f800000u;
            const float amax = nan_seen ? 0.f : __uint_as_float(top);
            const float lse2 = any_bad ? __uint_as_float(0x7fc00000u) : big + log2f(l_tot);
            if constexpr (SOLO) {
                // no merge: the rows go out as they are, by its rules: a NaN or an infinity spoils its row (the 16-bit format
                // holds neither), and no score above -inf leaves no log-sum-exp either
                if (row < p.rows) {
                    const int R = row, node = (int)__umulhi((uint32_t)R << 8, p.g_magic), h = g_e * p.G + R - node * p.G;
                    const bool nan = any_bad || nan_seen || amax == INFINITY || lse2 != lse2;
                    uint32_t *dst = (uint32_t *)((uint16_t *)p.out + (int64_t)b_e * p.o_sb + (int64_t)node * p.o_st +
                                                 (int64_t)h * p.o_sh + 4 * c0);
#pragma unroll
                    for (int q = 0; q < CPT / 4; ++q)
                        *(uint2 *)(dst + 2 * q) = nan ? make_uint2(0x7fc07fc0u, 0x7fc07fc0u)
                                                      : make_uint2(q8_pack_bf16(acc[4 * q], acc[4 * q + 1]), q8_pack_bf16(acc[4 * q + 2], acc[4 * q + 3]));
                    if (p.lse && x_e % TPR == 0)
                        p.lse[(int64_t)b_e * p.lse_sb + (int64_t)h * p.lse_sh + (int64_t)node * p.lse_st] =
                            lse2 == -INFINITY ? __uint_as_float(0x7fc00000u) : lse2 * 0.6931471805599453f;
                }
            } else if (row < p.rows) {
                float scale, to_q;
                ta_q15_scale(amax, nan_seen, scale, to_q);
                const int64_t wrow = ta_ws_row(p, slot_e, 0, row);
                uint32_t *dst = (uint32_t *)(ta_part_row(p, wrow) + 8 * c0);
#pragma unroll
                for (int q = 0; q < CPT / 4; ++q)
                    *(uint2 *)(dst + 2 * q) = make_uint2(ta_q15_pack(acc[4 * q], acc[4 * q + 1], to_q),
                                                         ta_q15_pack(acc[4 * q + 2], acc[4 * q + 3], to_q));
                // (a NaN log-sum-exp poisons the row in the merge)
                if (x_e % TPR == 0)
                    *(float2 *)&p.ws_lse[2 * wrow] = make_float2(lse2, scale);
            }
        }
        if (any_bad && x_e == 0)
            ta_raise(p, any_bad);
        q8_lds_barrier();                                      // the rings are free for the next item
    }
}

template <int DH, int NW, int OCC, int MODE>
static hipError_t launch_q8(const TAQ8Params &p, hipStream_t stream, int dev)
{
    const size_t smem = q8_smem<DH, NW, OCC, MODE>(p.B);
    static_assert(OCC * Q8Shape<DH, NW, OCC>::FIXED <= 160 * 1024, "OCC workgroups per compute unit");
    if (smem > 160 * 1024)
        return hipErrorInvalidValue;
    static bool attr_set[64] = {};      // per device and instance; setting it twice is harmless
    if (!attr_set[dev]) {
        hipError_t e = hipFuncSetAttribute((const void *)ta_q8_kv_kernel<DH, NW, OCC, MODE>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess)
            return e;
        attr_set[dev] = true;
    }
    hipLaunchKernelGGL((ta_q8_kv_kernel<DH, NW, OCC, MODE>), dim3(MODE == Q8_SOLO ? p.B * p.Hkv : p.n_wg), dim3(64 * NW), smem, stream, TA_SCHED_ARGS(p), p);
    return hipGetLastError();
}

hipError_t ta_launch_q8_mfma(const TAQ8Params &p, hipStream_t stream, int dev)
{
    if (dev < 0 || dev >= 64)
        return hipErrorInvalidDevice;
    if (p.ks_rows != 32 || p.rows > 32 || (!p.solo && p.rows_grp != p.rows) || !p.part_q15 || p.ls != 2 || !p.is_bf16 || p.direct)
        return hipErrorInvalidValue;
    auto rows = [&](auto dh) {
        constexpr int D = decltype(dh)::value;
        if (p.solo)
            return p.solo == TA_SOLO_PAIR ? launch_q8<D, 4, 2, Q8_SOLO>(p, stream, dev) : launch_q8<D, 8, 1, Q8_SOLO>(p, stream, dev);
        return launch_q8<D, 8, 1, Q8_CUT>(p, stream, dev);
    };
    if (p.D == 128)
        return rows(std::integral_constant<int, 128>{});
    return p.D == 64 ? rows(std::integral_constant<int, 64>{}) : hipErrorInvalidValue;
}
