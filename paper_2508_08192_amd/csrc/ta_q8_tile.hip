// KV pass over the 8-bit cache for many query rows, and for fp32 queries (gfx950): head_dim 64 or 128, fp32 accumulation.
//
// A workgroup of NW waves (eight, or four of which two share a compute unit) keeps 32 RBW rows (64, 128 or 256) of one (request, KV
// head) and walks its share in tiles of 16 NW tokens.  The codes of a tile become bf16 values once per workgroup: every wave has
// its sixteen tokens' codes and scales on the way into registers for two tiles, turns them into values (scales and all: a power of two
// leaves them exact) on their way into LDS one tile ahead, and then multiplies its 32 rows with its part of the tile that all have written:
// wave w has rows 32 (w % RBW) .., and of the tile's runs of 32 tokens those that are w / RBW modulo NW / RBW.  Two tiles
// lie in LDS, one barrier per tile.
//
//     S^T[token, row] = K . Q^T ;  O^T[d, row] += V^T . P^T       (as in ta_mfma_ks.hip, on v_mfma_f32_32x32x16_bf16)
//
// Where every wave converts for itself (ta_q8_attn.hip) a run of 32 tokens costs it 64 conversions beside 16 products of 32 cycles,
// and the loads' addresses on top.  The tokens of the tree follow the prefix without a gap, in the same tiles; a row's mask
// is laid over the positions.
//
// An fp32 query is the sum of three bf16 numbers, exactly (8 bits of its 24 each), and so is a probability; K and V are bf16 as they
// are, so three matrix products give what one in fp32 would.  Their first terms of Q stay in registers, the others in LDS, which
// leaves room for tiles of 64 tokens at head_dim 128.  Not taken: the fp32 matrix instruction, a sixteenth of the bf16 one's rate.
//
// What bounds it, and what it takes (with the merge):
//   256 rows, 4 requests of 131072 tokens, 8 KV heads: 590 us, 930 TFLOP/s, where a square product of 8192 in bf16 reaches 1200;
//       the matrix cores (46 % of all cycles) and the vector units (53 %) in turn, at some 1.9 GHz; a priority for one of two waves, or
//       none for either, changes nothing.
//   64 rows, 32 requests of 512 to 8192 tokens: 79 us, 3.8 TB/s; the chain of a tile's steps in each of two waves per SIMD (a tile of 64
//       tokens takes a wave some 3000 cycles, 900 of them conversions and 1450 scores, exponentials and products); it is hardly
//       faster when all pages lie in the L2.
// Not faster: waves of 64 rows, which read half as many bytes of K and V from LDS, but have no registers left for all of Q (657 us
// for the first); two groups of waves that take turns at the matrix cores with a barrier at every turn (695); conversions placed
// between the products of the scores (610, and 87 for the second).
#include <type_traits>

#include "ta_q8.h"

typedef __bf16 qt_bf16x8 __attribute__((ext_vector_type(8)));
typedef float qt_f32x16 __attribute__((ext_vector_type(16)));
typedef short qt_s4 __attribute__((ext_vector_type(4)));
typedef short qt_s8 __attribute__((ext_vector_type(8)));
typedef uint32_t qt_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t qt_u32x4_8 __attribute__((ext_vector_type(4), aligned(8)));     // (outputs start on 8 bytes)

#define QT_LENS 256                              // batches of up to this many requests keep their lengths in LDS

__device__ __forceinline__ float qt_swap_max(float x)      // over the two lanes that share a query row
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ uint32_t qt_row16_max(uint32_t x)           // over sixteen neighbouring lanes
{
    auto up = [&](uint32_t y) { x = y > x ? y : x; };
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));     // lanes 1 0 3 2 of every four
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));     // 2 3 0 1
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));    // mirrored within eight
    up((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));    // rotated by eight within sixteen
    return x;
}

__device__ __forceinline__ void qt_lds_barrier()           // (loads into registers stay in flight)
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ uint32_t qt_infinite(uint32_t x)            // is one of two bf16 numbers infinite (or none)?
{
    return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}

template <int DH, int NW, bool F32>
struct QtShape {
    static constexpr int TOKENS = F32 && DH == 128 ? 64 : 16 * NW;   // of a tile
    static constexpr int ROW = 2 * DH;                     // bytes of a token row in LDS
    static constexpr int TILE = TOKENS * ROW;             // of a tile's K (or V)
    static constexpr int BUF = 2 * TILE;
    static constexpr int LPR = DH / 16;                    // lanes of a row as it is loaded
    static constexpr int RPL = 64 / LPR;                   // rows of a load
    static constexpr int TPW = TOKENS / NW;                // tokens that a wave loads
    static constexpr int NL = TPW / RPL;                   // loads of those of K (or V)
    static constexpr int STAGE = 32 * DH * 4;              // a wave's results at the end
    static constexpr int QL = F32 ? 2 * 128 * ROW : 0;     // second and third terms of the queries
    static constexpr int TILES = 2 * BUF + QL;
    static constexpr int FIXED = TILES + 4 * NW * 2 * 32 + 4 * 8 + 8 + 8;
    static_assert(NW * STAGE <= TILES, "results are staged in the tiles' place");
};

enum { QT_CUT, QT_SOLO };                                  // see ta_q8_attn.hip

template <int DH, int NW, bool F32, int MODE>
static constexpr size_t qt_smem(int B)
{
    return QtShape<DH, NW, F32>::FIXED + (MODE == QT_SOLO || B <= TA_WAVE ? 0 : sizeof(int) * (B + 2 + (B <= QT_LENS ? 2 * B : 0)));
}

// Two numbers' upper halves: their leading eight bits as bf16, exact, and what the numbers lose by it.
__device__ __forceinline__ uint32_t qt_split(float &x, float &y)
{
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    x -= __uint_as_float(a & 0xffff0000u);
    y -= __uint_as_float(b & 0xffff0000u);
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

template <int DH, int RBW, int NW, int MODE, bool F32>
__global__ __launch_bounds__(64 * NW, 2) void ta_q8_tile_kernel(TA_SCHED_PARAMS, TAQ8Params p)
{
    const TASched sc = TA_SCHED;
    using C = QtShape<DH, NW, F32>;
    constexpr bool SOLO = MODE == QT_SOLO;
    constexpr int KW = NW / RBW, NR = C::TOKENS / 32 / KW, WSTEP = F32 ? 1 : RBW;      // waves that share rows, runs of a tile for each of them, from one to the next
    constexpr int TERMS = F32 ? 3 : 1;                                   // bf16 numbers whose sum is a query's or a probability's
    constexpr int NKK = DH / 16, NDB = DH / 32, NL = C::NL, ROWS = 32 * RBW;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *const stat = (float *)(smem + C::TILES);                      // [NW][2][32]: reference and sum
    int *const wbad = (int *)(stat + NW * 2 * 32);                       // [NW]: TA_STATUS_* bits a wave has met
    unsigned long long *const nan_nodes = (unsigned long long *)(wbad + 8);   // nodes whose values hold a NaN
    int *const cum = (int *)(nan_nodes + 2);                             // more than 64 requests: [B + 1] schedule
    int *const lens = cum + sc.B + 1, *const starts = lens + sc.B;       // and, up to QT_LENS, lengths and window starts

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = blockIdx.x, row0 = blockIdx.y * ROWS;                  // first of the workgroup's query rows
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rb = F32 ? wave / KW : wave % RBW, kg = F32 ? wave % KW : wave / RBW;
    const int r32 = lane & 31, hf = lane >> 5;
    // schedule, as in ta_q8_attn.hip
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
            total = sc.Hkv * ta_build_schedule(sc, cum, sc.B <= QT_LENS ? lens : nullptr, sc.B <= QT_LENS ? starts : nullptr);
        }
        ta_wg_range(sc, total, w, t, t_end);
        t = __builtin_amdgcn_readfirstlane(t);
        t_end = __builtin_amdgcn_readfirstlane(t_end);
    }
    const int rows_here = min(ROWS, p.rows - row0);
    // (fp32: a wave without rows only loads and converts for the others.  128 requests with 8 rows 120 us, 164 with products of rows
    // that nobody asked for; with no more than 64 rows those that have any lie on SIMDs of their own.)
    const int n_runs = !F32 || 32 * rb < rows_here ? NR : 0;
    const float c = p.scale_log2e;
    const bool paged = p.page_table != nullptr;
    // 16-byte slots of a row in LDS: K slot s of row r holds chunk s ^ kx(r), V slot s chunk s ^ 2 vx(r) (see ta_mfma_ks.hip).  At
    // head_dim 128 the chunks from the eighth on are swapped in pairs, so that the lanes of a row, which write every other chunk at a
    // time, spread over all banks: of a pass's LDS cycles 30 % were conflicts, now none are, and a call takes 1 % less.
    auto kx = [](int r) { return DH == 64 ? (r >> 1) & 7 : r & 15; };
    auto vx = [](int r) { return DH == 64 ? 2 * ((r >> 1) & 1) + ((r >> 2) & 1) : 2 * (r & 3) + ((r >> 2) & 1); };
    const int kf_at = r32 * C::ROW + ((hf ^ kx(r32)) << 4);
    const int vtk = 4 * hf + ((lane >> 2) & 3);
    const int vf_at = vtk * C::ROW + (lane & 3) * 8 + ((((lane >> 4) & 1) ^ vx(vtk)) << 5);
    const int lrow = lane / C::LPR, lchunk = lane % C::LPR;              // as a lane loads: its row of a load's, its sixteen columns
    const bool s_is_v = lane % (2 * C::TPW) >= C::TPW;                   // of two lanes a token's scales
    const uint32_t s_step = (uint32_t)(s_is_v ? p.vs_ss : p.ks_ss), s_lane = lane % C::TPW * s_step;
    const uint32_t k_lane = lrow * (uint32_t)p.k_ss + 16u * lchunk, v_lane = lrow * (uint32_t)p.v_ss + 16u * lchunk;
    int kw_at[NL][2], vw_at[NL][2];                                      // where their two halves go
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = C::TPW * wave + i * C::RPL + lrow;
            kw_at[i][h] = row * C::ROW + (((2 * lchunk + h) ^ kx(row) ^ (lchunk >> 2)) << 4);
            vw_at[i][h] = row * C::ROW + (((2 * lchunk + h) ^ (2 * vx(row)) ^ (lchunk >> 2)) << 4);
        }

    typedef __attribute__((address_space(3))) char *lds_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_t)smem;              // (zero, but the compiler adds it to every address that it does not see)
    // ---- the current item: list (b, g), tokens at positions [first, end) of the request, those from L on being the tree's
    int b = -1, g = 0, slot = 0, L = 0, first = 0, end = 0, base = 0, n_t = 0, bad = 0;
    auto next_item = [&]() {
        while (t < t_end) {
            int n_b, j0, j1, S;
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
                    L = __builtin_amdgcn_readfirstlane(sc.B <= QT_LENS ? lens[b] : sc.seq_lens[(int64_t)b * sc.sl_s]);
                    S = __builtin_amdgcn_readfirstlane(sc.B <= QT_LENS ? starts[b] : ta_kv_start(sc, b));
                }
            }
            b = __builtin_amdgcn_readfirstlane(b);
            g = __builtin_amdgcn_readfirstlane(g);
            L = __builtin_amdgcn_readfirstlane(L);
            S = __builtin_amdgcn_readfirstlane(S);
            j0 = __builtin_amdgcn_readfirstlane(j0);
            j1 = __builtin_amdgcn_readfirstlane(j1);
            const bool ok = ta_request_ok(sc, L, S);
            bad = ok ? 0 : TA_STATUS_BAD_SEQLEN;
            const int tile0 = ok ? S / TA_TILE : 0;
            const bool has_tree = j1 == n_b;
            first = has_tree && j0 == n_b - 1 ? L : max((tile0 + j0) * TA_TILE, S);
            end = has_tree ? L + sc.T : min((tile0 + j1) * TA_TILE, L);
            if (!ok) {                                                 // (its loads, which nobody uses, go to the first token of a page)
                first = 0;
                end = 1;
            }
            base = first & ~31;
            n_t = !ok ? 0 : (end - base + C::TOKENS - 1) / C::TOKENS;
            return true;
        }
        return false;
    };

    struct Raw {                                           // a wave's sixteen tokens of a tile
        qt_u32x4 k[NL], v[NL];
        uint32_t scale;                                    // lane l: K's of token l, V's of token l - TPW
    };

    while (next_item()) {
        // ---- what the start of an item needs: Q, the tree, page ids of this wave's tokens (lane l: tile pg_base + l)
        int pg = 0, pg_base = 0;
        auto load_pages = [&](int from) {
            const int pos = base + (from + lane) * C::TOKENS + C::TPW * wave;
            const int at = min(max(pos, first), end - 1);
            return p.page_table[(int64_t)b * p.pt_sb + (at >> p.ps_shift)];
        };
        auto checked = [&](int id) {                       // a page id as an address: one outside the cache is reported
            if (!ta_page_ok(p, id)) {
                bad |= TA_STATUS_BAD_PAGE;
                id = 0;
            }
            return id;
        };
        unsigned long long tmask = ~0ull;
        if (!bad && paged)
            pg = load_pages(0);
        uint4 qf[NKK];
        uint4 *const ql = (uint4 *)(smem + 2 * C::BUF) + rb * NKK * TA_WAVE + lane;
        {
            // rows past the group's end repeat its first row (their results are never stored)
            const int row = rb * 32 + r32, R = row0 + (row < rows_here ? row : 0);
            const int node = (int)__umulhi((uint32_t)R << 8, p.g_magic);              // R / G
            const int64_t at = (int64_t)b * p.q_sb + (int64_t)node * p.q_st + (int64_t)(g * p.G + R - node * p.G) * p.q_sh + 8 * hf;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) {
                if constexpr (F32) {
                    const float4 x0 = *(const float4 *)((const float *)p.q + at + 16 * kk), x1 = *(const float4 *)((const float *)p.q + at + 16 * kk + 4);
                    float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        const uint4 y = make_uint4(qt_split(x[0], x[1]), qt_split(x[2], x[3]), qt_split(x[4], x[5]), qt_split(x[6], x[7]));
                        if (t == 0)
                            qf[kk] = y;
                        else if (kg == 0)                              // (the waves that share rows share these)
                            ql[((t - 1) * RBW * NKK + kk) * TA_WAVE] = y;
                    }
                } else {
                    qf[kk] = *(const uint4 *)((const uint16_t *)p.q + at + 16 * kk);
                }
            }
        }
        int parent = 0;
        unsigned long long gmask = 0;
        const bool tree_here = !bad && end > L;
        if (tree_here && lane < sc.T) {
            if (p.masks_in)
                gmask = ta_given_mask(p, b, lane);
            else
                parent = p.parent[(int64_t)b * p.par_sb + lane];
        }
        if (!bad && paged)
            pg = checked(pg);
        const uint8_t *const kgp = (const uint8_t *)p.k + (int64_t)g * p.k_sh, *const vgp = (const uint8_t *)p.v + (int64_t)g * p.v_sh;
        const uint8_t *const ksp = p.ks + (int64_t)g * p.ks_sh, *const vsp = p.vs + (int64_t)g * p.vs_sh;

        // The loads of a tile, the same number whatever the tile, so that a wait can leave the next one's in flight: tokens outside
        // [first, end) are read as the nearest that is in it, and the tiles behind the last as the last token.
        auto load_tile = [&](int j, Raw &x) {
            if (paged && j - pg_base >= TA_WAVE) {
                pg_base = j;                                           // (waits)
                pg = checked(load_pages(pg_base));
            }
            const int pos0 = base + j * C::TOKENS + C::TPW * wave, at0 = min(max(pos0, first), end - 1) & -C::TPW;
            const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(paged ? pg : b, paged ? j - pg_base : 0);
            const uint32_t sl0 = (uint32_t)(paged ? at0 & (p.ps - 1) : at0);
            // (bases are scalars, and the lanes' offsets fit in 32 bits: the host has seen to it)
            const uint8_t *kb = kgp + (uint64_t)page * (uint32_t)p.k_sp + (uint64_t)sl0 * (uint32_t)p.k_ss;
            const uint8_t *vb = vgp + (uint64_t)page * (uint32_t)p.v_sp + (uint64_t)sl0 * (uint32_t)p.v_ss;
            const uint64_t ko = (uint64_t)page * (uint32_t)p.ks_sp + (uint64_t)sl0 * (uint32_t)p.ks_ss;
            const uint64_t vo = (uint64_t)page * (uint32_t)p.vs_sp + (uint64_t)sl0 * (uint32_t)p.vs_ss;
            uint32_t so = s_lane, koff[NL], voff[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                koff[i] = k_lane + i * C::RPL * (uint32_t)p.k_ss;
                voff[i] = v_lane + i * C::RPL * (uint32_t)p.v_ss;
            }
            if (pos0 < first || pos0 + C::TPW > end) {
                const int hi = min(end - 1 - at0, C::TPW - 1), lo = pos0 >= end ? hi : max(first - at0, 0);
                so = (uint32_t)min(max(lane % C::TPW, lo), hi) * s_step;
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const uint32_t r = (uint32_t)min(max(i * C::RPL + lrow, lo), hi);
                    koff[i] = r * (uint32_t)p.k_ss + 16u * lchunk;
                    voff[i] = r * (uint32_t)p.v_ss + 16u * lchunk;
                }
            }
            x.scale = (s_is_v ? vsp + vo : ksp + ko)[so];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                x.k[i] = __builtin_nontemporal_load((const qt_u32x4 *)(kb + koff[i]));
                x.v[i] = __builtin_nontemporal_load((const qt_u32x4 *)(vb + voff[i]));
            }
        };
        // into the tile at byte `buf` of LDS
        auto write_tile = [&](int j, int buf, Raw &x) {
            if (j >= n_t)
                return;
            const int pos0 = base + j * C::TOKENS + C::TPW * wave;
            const bool edge = pos0 < first || pos0 + C::TPW > min(L, end);
            const int scale = (int)__float_as_uint(q8_scale(x.scale));   // (one conversion per token and tensor, then sent to those who need it)
            float kscale[NL], vscale[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                kscale[i] = __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(4 * lrow + 4 * i * C::RPL, scale));
                vscale[i] = __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(4 * lrow + 4 * (C::TPW + i * C::RPL), scale));
            }
            if (edge) {
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    // tokens of others are zeros; a NaN among a node's values counts only for rows that attend to it, so it is noted
                    // and taken out of the product
                    const int pos = pos0 + i * C::RPL + lrow;
                    const bool mine = pos >= first && pos < end;
                    if (!mine) {
                        x.k[i] = qt_u32x4{0u, 0u, 0u, 0u};
                        kscale[i] = 1.f;
                    }
                    uint32_t nan = vscale[i] != vscale[i] ? 1u : 0u;
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        nan |= ((x.v[i][n] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                    if (vscale[i] >= 0x1p120f) {           // (a value past the largest number counts as one that is none)
#pragma unroll
                        for (int n = 0; n < 4; ++n)
                            nan |= qt_infinite(q8_bf16_2<false>(x.v[i][n], vscale[i])) | qt_infinite(q8_bf16_2<true>(x.v[i][n], vscale[i]));
                    }
                    if (mine && pos >= L && nan)
                        atomicOr(nan_nodes, 1ull << (pos - L));
                    if (!mine || (pos >= L && nan)) {
                        x.v[i] = qt_u32x4{0u, 0u, 0u, 0u};
                        vscale[i] = 1.f;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    typedef __attribute__((address_space(3))) qt_u32x4 *lds_u4;
                    const uint32_t k0 = x.k[i][2 * h], k1 = x.k[i][2 * h + 1], v0 = x.v[i][2 * h], v1 = x.v[i][2 * h + 1];
                    *(lds_u4)(uintptr_t)(lds0 + kw_at[i][h] + buf) =
                        qt_u32x4{q8_bf16_2<false>(k0, kscale[i]), q8_bf16_2<true>(k0, kscale[i]), q8_bf16_2<false>(k1, kscale[i]), q8_bf16_2<true>(k1, kscale[i])};
                    *(lds_u4)(uintptr_t)(lds0 + vw_at[i][h] + buf + C::TILE) =
                        qt_u32x4{q8_bf16_2<false>(v0, vscale[i]), q8_bf16_2<true>(v0, vscale[i]), q8_bf16_2<false>(v1, vscale[i]), q8_bf16_2<true>(v1, vscale[i])};
                }
            }
        };

        Raw even = {}, odd = {};
        load_tile(0, even);
        load_tile(1, odd);
        if (tid == 0)
            *nan_nodes = 0ull;
        qt_f32x16 o[NDB];
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[db][i] = 0.f;
        float m_run = -INFINITY, l_run = 0.f;
        if (tree_here) {
            // lane i walks up from node i
            unsigned long long m = 0;
            bool wrong = false;
            if (p.masks_in) {
                m = gmask;
                wrong = lane < sc.T && !ta_given_mask_ok(m, lane);
            } else {
                int cur = lane < sc.T ? lane : -1;
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
            const int row = rb * 32 + r32, node = p.q_off + (int)__umulhi((uint32_t)(row0 + row) << 8, p.g_magic);
            const uint32_t m_lo = __shfl((uint32_t)m, node & 63, TA_WAVE), m_hi = __shfl((uint32_t)(m >> 32), node & 63, TA_WAVE);
            if (row < rows_here)
                tmask = ((unsigned long long)m_hi << 32) | m_lo;
        }
        qt_lds_barrier();                                  // (nan_nodes is zero, and the tiles' place is free)
        write_tile(0, 0, even);
        load_tile(2, even);
        qt_lds_barrier();

        // 32 tokens from position pos0 on, at row `at` of the tile in LDS
        auto run = [&](int tile, int at, int pos0) {
            // ---- S^T = K . Q^T
            qt_f32x16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            uint32_t ka = lds0 + at * C::ROW + kf_at, va = lds0 + at * C::ROW + vf_at;
            asm volatile("" : "+v"(ka), "+v"(va));         // (one operation per address, where addresses that are kept would not fit in registers)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) {
                const qt_u32x4 kf = *(const __attribute__((address_space(3))) qt_u32x4 *)(uintptr_t)((ka ^ (kk << 5) ^ (kk / 4 << 4)) + tile);
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) {
                    const uint4 qk = t == 0 ? qf[kk] : ql[((t - 1) * RBW * NKK + kk) * TA_WAVE];
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(qt_bf16x8, kf), __builtin_bit_cast(qt_bf16x8, qk), s, 0, 0, 0);
                }
            }
            // ---- V fragments: the first half is requested here and arrives under the softmax, the second under the products of the first
            typedef __attribute__((address_space(3))) qt_s4 *lds_s4;
            auto v_frag = [&](int kb, int db) {
                const uint32_t a = (va ^ (db << 6) ^ (db / 2 << 4)) + tile + C::TILE + kb * 16 * C::ROW;
                const qt_s4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)a);
                const qt_s4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)(a + 8 * C::ROW));
                return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            qt_s8 vf[NDB];
#pragma unroll
            for (int db = 0; db < NDB; ++db)
                vf[db] = v_frag(0, db);
            __builtin_amdgcn_s_setprio(0);
            // ---- scores of tokens that do not exist, or that are no ancestors, become -inf
            if (pos0 < first || pos0 + 32 > min(L, end)) {
                uint32_t mm = 0;
                if (pos0 < L) {
                    const int n = min(L, end) - pos0;                  // prefix tokens from pos0 on
                    mm = n >= 32 ? ~0u : n > 0 ? (1u << n) - 1u : 0u;
                    if (pos0 < first)
                        mm &= first - pos0 >= 32 ? 0u : ~((1u << (first - pos0)) - 1u);
                }
                if (end > L) {
                    const unsigned long long tm = sc.T >= 64 ? tmask : tmask & ((1ull << sc.T) - 1ull);
                    const int up = L - pos0;
                    mm |= up >= 32 ? 0u : up >= 0 ? (uint32_t)tm << up : (uint32_t)(tm >> -up);
                }
                mm >>= 4 * hf;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((mm >> (8 * (i / 4) + (i % 4))) & 1u))
                        s[i] = -INFINITY;
            }
            // ---- running softmax (the reference moves only when a score exceeds it by more than 2^4: see ta_mfma_ks.hip)
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i)
                top = __builtin_elementwise_maximum(top, s[i]);          // (of a NaN a NaN, which moves nothing: such a row is NaN anyway)
            top *= c;
            if (__any(top > m_run + (SOLO ? 0.f : 4.f))) {
                const float m_new = fmaxf(m_run, qt_swap_max(top));
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[db][i] *= alpha;
            }
            const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
            uint32_t pk[TERMS][8];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * i], c, neg_m)), e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], c, neg_m));
                sum[i & 1] += e0 + e1;
                if constexpr (F32) {
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        pk[t][i] = qt_split(e0, e1);
                } else {
                    pk[0][i] = q8_pack_bf16(e0, e1);
                }
            }
            l_run += sum[0] + sum[1];
            // ---- O^T += V^T . P^T
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                for (int db = 0; db < NDB; ++db) {
#pragma unroll
                    for (int t = TERMS - 1; t >= 0; --t) {
                        const uint4 pb = make_uint4(pk[t][4 * kb], pk[t][4 * kb + 1], pk[t][4 * kb + 2], pk[t][4 * kb + 3]);
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(qt_bf16x8, vf[db]), __builtin_bit_cast(qt_bf16x8, pb),
                                                                        o[db], 0, 0, 0);
                    }
                    if (kb == 0)
                        vf[db] = v_frag(1, db);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        };
        // (which of the two tiles in LDS is known where a step is compiled)
        auto step = [&](int j, auto even_step, Raw &next) {
            constexpr int BUF = decltype(even_step)::value ? 0 : C::BUF;
            write_tile(j + 1, C::BUF - BUF, next);
            load_tile(j + 3, next);
#pragma unroll 1
            for (int r = 0; r < n_runs; ++r) {
                const int at = 32 * (kg + KW * r), pos0 = base + j * C::TOKENS + at;
                if (pos0 < end && pos0 + 32 > first)
                    run(BUF, at, pos0);
            }
            qt_lds_barrier();
        };
#pragma unroll 1
        for (int j = 0; j < n_t; j += 2) {                 // (no way out in between: one more path here, and all waits are for everything)
            step(j, std::true_type{}, odd);
            step(j + 1, std::false_type{}, even);
        }

        // ---- results.  A wave that shares its rows with no other has all of them in registers.  Otherwise each wave stages its 32 x DH
        // block (16-byte chunk ch of row r at chunk ch ^ (r & 15)), and the threads add up those of the waves that share rows.
        constexpr bool ALONE = KW == 1 && !F32;
        {
            int wb = 0;
            if (__any(bad)) {
                for (int bit : {TA_STATUS_BAD_PARENT, TA_STATUS_BAD_SEQLEN, TA_STATUS_BAD_PAGE})
                    wb |= __any(bad & bit) ? bit : 0;
            }
            if (lane == 0)
                wbad[wave] = wb;
            if (tree_here && (tmask & *nan_nodes)) {
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[db][i] = __uint_as_float(0x7fc00000u);
            }
            if constexpr (!ALONE) {
                const float l_tot = l_run + __shfl_xor(l_run, 32, TA_WAVE);
                if (hf == 0) {
                    stat[(wave * 2 + 0) * 32 + r32] = m_run;
                    stat[(wave * 2 + 1) * 32 + r32] = l_tot;
                }
                float *stage = (float *)(smem + wave * C::STAGE);
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const int ch = db * 8 + 2 * i4 + hf;
                        *(float4 *)(stage + r32 * DH + ((ch ^ (r32 & 15)) << 2)) =
                            make_float4(o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]);
                    }
            }
        }
        qt_lds_barrier();
        int any_bad = 0;
#pragma unroll
        for (int k = 0; k < NW; ++k)
            any_bad |= wbad[k];
        if constexpr (ALONE) {
            const int row = rb * 32 + r32;
            const float l_tot = l_run + __shfl_xor(l_run, 32, TA_WAVE), inv = any_bad ? 0.f : 1.f / l_tot;
            uint32_t top = 0;                              // (bits of the row's largest magnitude, as below)
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    o[db][i] *= inv;
                    top = max(top, __float_as_uint(o[db][i]) & 0x7fffffffu);
                }
            top = max(top, (uint32_t)__shfl_xor((int)top, 32, TA_WAVE));
            const bool nan_seen = top > 0x7f800000u;
            const float amax = nan_seen ? 0.f : __uint_as_float(top);
            const float lse2 = any_bad ? __uint_as_float(0x7fc00000u) : m_run + log2f(l_tot);
            float scale, to_q;
            ta_q15_scale(amax, nan_seen, scale, to_q);
            const bool nan = any_bad || nan_seen || amax == INFINITY || lse2 != lse2;
            const int R = row0 + (row < rows_here ? row : 0), node = (int)__umulhi((uint32_t)R << 8, p.g_magic), h = g * p.G + R - node * p.G;
            const int64_t wrow = SOLO ? 0 : ta_ws_row(p, slot, 0, R);
            char *const dst = SOLO ? (char *)((uint16_t *)p.out + (int64_t)b * p.o_sb + (int64_t)node * p.o_st + (int64_t)h * p.o_sh)
                                   : ta_part_row(p, wrow);
            auto two = [&](float x, float y) { return SOLO ? (nan ? 0x7fc07fc0u : q8_pack_bf16(x, y)) : ta_q15_pack(x, y, to_q); };
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int p2 = 0; p2 < 2; ++p2) {
                    // the two halves of a row exchange columns: a lane then has eight in a row
                    const int e = 8 * p2;
                    const auto w0 = __builtin_amdgcn_permlane32_swap(two(o[db][e], o[db][e + 1]), two(o[db][e + 4], o[db][e + 5]), false, false);
                    const auto w1 = __builtin_amdgcn_permlane32_swap(two(o[db][e + 2], o[db][e + 3]), two(o[db][e + 6], o[db][e + 7]), false, false);
                    if (row < rows_here)
                        *(qt_u32x4_8 *)(dst + 2 * (32 * db + 16 * p2 + 8 * hf)) = qt_u32x4_8{w0[0], w1[0], w0[1], w1[1]};
                }
            if (row < rows_here && hf == 0) {
                if constexpr (!SOLO)
                    *(float2 *)&p.ws_lse[2 * wrow] = make_float2(lse2, scale);
                else if (p.lse)
                    p.lse[(int64_t)b * p.lse_sb + (int64_t)h * p.lse_sh + (int64_t)node * p.lse_st] =
                        lse2 == -INFINITY ? __uint_as_float(0x7fc00000u) : lse2 * 0.6931471805599453f;
            }
            if (any_bad && tid == 0)
                ta_raise(p, any_bad);
            qt_lds_barrier();                              // everything has been read
            continue;
        }
        constexpr int CPT = DH / 16;                       // columns of a thread: sixteen of them per row
#pragma unroll 1
        for (int row = tid / 16; row < ROWS; row += 4 * NW) {
            const int c0 = (tid % 16) * (CPT / 4), rr = row & 31, wv0 = F32 ? row / 32 * KW : row / 32;       // the first wave of its rows
            float mw[KW], big = -INFINITY;
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                mw[k] = stat[((wv0 + k * WSTEP) * 2 + 0) * 32 + rr];
                big = fmaxf(big, mw[k]);
            }
            float l_tot = 0.f, acc[CPT];
#pragma unroll
            for (int i = 0; i < CPT; ++i)
                acc[i] = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const float wgt = mw[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[k] - big);
                l_tot = fmaf(wgt, stat[((wv0 + k * WSTEP) * 2 + 1) * 32 + rr], l_tot);
#pragma unroll
                for (int q = 0; q < CPT / 4; ++q) {
                    const float4 x = *(const float4 *)(smem + (wv0 + k * WSTEP) * C::STAGE + (rr * DH + (((c0 + q) ^ (rr & 15)) << 2)) * 4);
                    acc[4 * q + 0] = fmaf(wgt, x.x, acc[4 * q + 0]);
                    acc[4 * q + 1] = fmaf(wgt, x.y, acc[4 * q + 1]);
                    acc[4 * q + 2] = fmaf(wgt, x.z, acc[4 * q + 2]);
                    acc[4 * q + 3] = fmaf(wgt, x.w, acc[4 * q + 3]);
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
            top = qt_row16_max(top);
            const bool nan_seen = top > 0x7f800000u;
            const float amax = nan_seen ? 0.f : __uint_as_float(top);
            const float lse2 = any_bad ? __uint_as_float(0x7fc00000u) : big + log2f(l_tot);
            if (row < rows_here) {
                if constexpr (SOLO) {
                    // (no merge: the rules are those of ta_q8_attn.hip)
                    const int R = row0 + row, node = (int)__umulhi((uint32_t)R << 8, p.g_magic), h = g * p.G + R - node * p.G;
                    const bool nan = any_bad || nan_seen || amax == INFINITY || lse2 != lse2;
                    const int64_t at = (int64_t)b * p.o_sb + (int64_t)node * p.o_st + (int64_t)h * p.o_sh + 4 * c0;
                    if constexpr (F32) {
                        const float qnan = __uint_as_float(0x7fc00000u);
#pragma unroll
                        for (int q = 0; q < CPT / 4; ++q)
                            *(float4 *)((float *)p.out + at + 4 * q) = any_bad || lse2 != lse2 ? make_float4(qnan, qnan, qnan, qnan)
                                : make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
                    } else {
                        uint32_t *dst = (uint32_t *)((uint16_t *)p.out + at);
#pragma unroll
                        for (int q = 0; q < CPT / 4; ++q)
                            *(uint2 *)(dst + 2 * q) = nan ? make_uint2(0x7fc07fc0u, 0x7fc07fc0u)
                                : make_uint2(q8_pack_bf16(acc[4 * q], acc[4 * q + 1]), q8_pack_bf16(acc[4 * q + 2], acc[4 * q + 3]));
                    }
                    if (p.lse && tid % 16 == 0)
                        p.lse[(int64_t)b * p.lse_sb + (int64_t)h * p.lse_sh + (int64_t)node * p.lse_st] =
                            lse2 == -INFINITY ? __uint_as_float(0x7fc00000u) : lse2 * 0.6931471805599453f;
                } else if constexpr (F32) {
                    const int64_t wrow = ta_ws_row(p, slot, 0, row0 + row);
                    float *dst = (float *)ta_part_row(p, wrow) + 4 * c0;
#pragma unroll
                    for (int q = 0; q < CPT / 4; ++q)
                        *(float4 *)(dst + 4 * q) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
                    if (tid % 16 == 0)
                        p.ws_lse[wrow] = lse2;
                } else {
                    float scale, to_q;
                    ta_q15_scale(amax, nan_seen, scale, to_q);
                    const int64_t wrow = ta_ws_row(p, slot, 0, row0 + row);
                    uint32_t *dst = (uint32_t *)(ta_part_row(p, wrow) + 8 * c0);
#pragma unroll
                    for (int q = 0; q < CPT / 4; ++q)
                        *(uint2 *)(dst + 2 * q) = make_uint2(ta_q15_pack(acc[4 * q], acc[4 * q + 1], to_q),
                                                             ta_q15_pack(acc[4 * q + 2], acc[4 * q + 3], to_q));
                    // (a NaN log-sum-exp poisons the row in the merge)
                    if (tid % 16 == 0)
                        *(float2 *)&p.ws_lse[2 * wrow] = make_float2(lse2, scale);
                }
            }
        }
        if (any_bad && tid == 0)
            ta_raise(p, any_bad);
        qt_lds_barrier();                                  // everything has been read
    }
}

template <int DH, int RBW, int NW, int MODE, bool F32>
static hipError_t launch_tile(const TAQ8Params &p, hipStream_t stream, int dev)
{
    const size_t smem = qt_smem<DH, NW, F32, MODE>(p.B);
    static_assert(qt_smem<DH, NW, F32, MODE>(TA_MAX_BATCH) <= 160 * 1024, "whatever the batch");
    static bool attr_set[64] = {};      // per device and instance; setting it twice is harmless
    if (!attr_set[dev]) {
        hipError_t e = hipFuncSetAttribute((const void *)ta_q8_tile_kernel<DH, RBW, NW, MODE, F32>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                           160 * 1024);
        if (e != hipSuccess)
            return e;
        attr_set[dev] = true;
    }
    hipLaunchKernelGGL((ta_q8_tile_kernel<DH, RBW, NW, MODE, F32>), dim3(MODE == QT_SOLO ? p.B * p.Hkv : p.n_wg, (p.rows + 32 * RBW - 1) / (32 * RBW)),
                       dim3(64 * NW), smem, stream, TA_SCHED_ARGS(p), p);
    return hipGetLastError();
}

hipError_t ta_launch_q8_tile(const TAQ8Params &p, hipStream_t stream, int dev)
{
    if (dev < 0 || dev >= 64)
        return hipErrorInvalidDevice;
    if (p.direct || (!p.solo && p.rows_grp != p.rows) || p.part_q15 != p.is_bf16 || p.ls != (p.is_bf16 ? 2 : 1) ||
        (!p.is_bf16 && p.ks_rows != 128))
        return hipErrorInvalidValue;
    auto with = [&](auto dh, auto rbw, auto f32) {
        constexpr int D = decltype(dh)::value, W = decltype(rbw)::value;
        constexpr bool F32 = decltype(f32)::value;
        if (p.solo == TA_SOLO_WIDE)
            return launch_tile<D, W, 8, QT_SOLO, F32>(p, stream, dev);
        if constexpr (W < 8 && !F32) {
            if (p.solo)
                return launch_tile<D, W, 4, QT_SOLO, F32>(p, stream, dev);
            if (p.waves == 4)
                return launch_tile<D, W, 4, QT_CUT, F32>(p, stream, dev);
        }
        return p.solo || p.waves != 8 ? hipErrorInvalidValue : launch_tile<D, W, 8, QT_CUT, F32>(p, stream, dev);
    };
    auto rows = [&](auto dh) {
        if (!p.is_bf16)
            return with(dh, std::integral_constant<int, 4>{}, std::true_type{});
        switch (p.ks_rows) {
        case 64: return with(dh, std::integral_constant<int, 2>{}, std::false_type{});
        case 128: return with(dh, std::integral_constant<int, 4>{}, std::false_type{});
        case 256: return with(dh, std::integral_constant<int, 8>{}, std::false_type{});
        default: return hipErrorInvalidValue;
        }
    };
    if (p.D == 128)
        return rows(std::integral_constant<int, 128>{});
    return p.D == 64 ? rows(std::integral_constant<int, 64>{}) : hipErrorInvalidValue;
}
