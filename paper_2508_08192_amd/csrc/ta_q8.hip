// Rotary positions and the ways into, out of and within the 8-bit cache.  All of it moves bytes; the arithmetic beside them (a
// sine and a cosine per token and pair of columns, shared by all heads; a maximum per row) is kept off the way of the loads.
#include "ta_q8.h"

#define ROWS_THREADS 256
#define ROWS_TOKENS 8                       // most tokens of a workgroup (see tokens_per_group)

// Depth of the tree's node `lane` (a root's is 0), in every lane below T.  Each step doubles the distance looked up from every
// node at once: six reach past any path of 64 nodes, so a node that still has an ancestor then lies on a cycle.
__device__ __forceinline__ int rows_depth(const TARows &a, int b, int lane, bool &bad)
{
    if (a.masks_in) {
        unsigned long long m = 0;
        if (lane < a.T) {
            m = a.masks_in[(int64_t)b * a.masks_sb + lane];
            m = a.T >= 64 ? m : m & ((1ull << a.T) - 1ull);
        }
        bad = __any(lane < a.T && !((m >> lane) & 1ull));
        return __popcll(m) - 1;
    }
    int up = lane < a.T ? a.parent[(int64_t)b * a.par_sb + lane] : -1;
    bool wrong = up >= a.T;
    up = wrong || up < 0 ? -1 : up;
    int depth = up >= 0 ? 1 : 0;
#pragma unroll
    for (int s = 0; s < 6; ++s) {
        const int d = __shfl(depth, up & 63, TA_WAVE), u = __shfl(up, up & 63, TA_WAVE);
        if (up >= 0) {
            depth += d;
            up = u;
        }
    }
    bad = __any(wrong || up >= 0);
    return depth;
}

// cos and sin of position * frequency, times the amplitude.  The angle is reduced to a part of a turn in 64 bits: at position
// 10^6 a 32-bit product would be off by up to 0.03.
__device__ __forceinline__ float2 rows_turn(double pos, float freq, float amplitude)
{
    const double k = 0.15915494309189533577, angle = pos * (double)freq;
    float s, c;
    sincospif(2.f * (float)fma(angle, k, -rint(angle * k)), &s, &c);
    return make_float2(c * amplitude, s * amplitude);
}

// (which product is rounded is said here, so that every kernel gives the same bits)
__device__ __forceinline__ void rows_rotate(float &x, float &y, float2 t)
{
    const float u = fmaf(x, t.x, -(y * t.y)), w = fmaf(y, t.x, x * t.y);
    x = u;
    y = w;
}

struct RowsPlace {
    int64_t page;                           // -1: not written
    int64_t slot;
};

__device__ __forceinline__ RowsPlace rows_place(const TARows &a, int b, int pos)
{
    RowsPlace r = {b, pos};
    if (a.page_table) {
        const int k = pos / a.ps;
        r.page = a.page_table[(int64_t)b * a.pt_sb + k];
        r.slot = pos - k * a.ps;
        if (r.page < 0 || r.page >= a.n_pages)
            r.page = -1;
    }
    return r;
}

// A row of every token (query, key or value head): where it comes from and goes to, but for the token.  The strides' unit is a byte.
struct RowsHead {
    int kind;                               // 0 query, 1 key, 2 value
    const char *src;
    int64_t src_st;
    char *dense;                            // rotated rows; null: into the cache
    int64_t dense_st;
    char *codes;
    int64_t code_sp, code_ss;
    uint8_t *scale;
    int64_t scale_sp, scale_ss;
};

template <bool BF16, bool QUANT>
__device__ __forceinline__ RowsHead rows_head(const TARows &a, int b, int y)
{
    constexpr int ES = BF16 ? 2 : 4;
    RowsHead r = {};
    r.kind = y < a.Hq ? 0 : y < a.Hq + a.Hkv ? 1 : 2;
    const int64_t h = r.kind == 0 ? y : r.kind == 1 ? y - a.Hq : y - a.Hq - a.Hkv;
    if (r.kind == 0) {
        r.src = (const char *)a.q + (b * a.q_sb + h * a.q_sh) * ES;
        r.src_st = a.q_st * ES;
        r.dense = (char *)a.q_out + (b * a.qo_sb + h * a.qo_sh) * ES;
        r.dense_st = a.qo_st * ES;
    } else if (r.kind == 1) {
        r.src = (const char *)a.k + (b * a.k_sb + h * a.k_sh) * ES;
        r.src_st = a.k_st * ES;
        if (QUANT) {
            r.codes = (char *)a.kc + h * a.k_shc;
            r.code_sp = a.k_sp;
            r.code_ss = a.k_ss;
            r.scale = a.ks + h * a.ks_sh;
            r.scale_sp = a.ks_sp;
            r.scale_ss = a.ks_ss;
        } else {
            r.dense = (char *)a.k_out + (b * a.ko_sb + h * a.ko_sh) * ES;
            r.dense_st = a.ko_st * ES;
        }
    } else {
        r.src = (const char *)a.v + (b * a.v_sb + h * a.v_sh) * ES;
        r.src_st = a.v_st * ES;
        r.codes = (char *)a.vc + h * a.v_shc;
        r.code_sp = a.v_sp;
        r.code_ss = a.v_ss;
        r.scale = a.vs + h * a.vs_sh;
        r.scale_sp = a.vs_sp;
        r.scale_ss = a.vs_ss;
    }
    return r;
}

// How a lane's columns pair up.
enum { ROWS_KEEP, ROWS_HALVES, ROWS_NEIGHBOURS };      // not at all; column j with j + R/2; 2j with 2j + 1

// Rotated (TURN) queries and keys to dense rows, or keys (rotated or not) and values into the cache (QUANT).  A lane holds sixteen
// columns of a row in two runs of eight, half of the rotated (or of the other) columns apart: each load and store of the lanes of a
// row is then one piece of memory, and columns that pair up across the halves meet in one lane.  The LPR lanes of a row find its
// maximum among themselves.  A thread keeps its head and goes from token to token, ROWS_AHEAD of them requested at a time.
// What bounds it: bytes in flight, and the round trips of a workgroup's start (length and tree, then the page).  8000 tokens of 40 heads
// rotated: 38 us, 4.3 TB/s read and written, where a copy reaches 5.4 (31 us when the rows lie in the caches); 4 prompts of 4001
// tokens, 8 KV heads, quantised: 25 us, 4.0 TB/s; 32 requests of 16 tokens, 48 heads, rotated and written: 8 us.
constexpr int ROWS_AHEAD = 4;

template <bool BF16, int TURN, bool QUANT, int LPR>
__global__ __launch_bounds__(ROWS_THREADS) void ta_rows_kernel(TARows a)
{
    constexpr int V = BF16 ? 1 : 2, ES = BF16 ? 2 : 4;     // 16-byte loads of eight columns, bytes of an element
    constexpr int RPP = ROWS_THREADS / LPR;                // rows at a time
    __shared__ float2 turn[TURN ? ROWS_TOKENS : 1][TURN ? TA_MAX_HEAD_DIM / 2 : 1];
    __shared__ RowsPlace place[ROWS_TOKENS];
    __shared__ int depths[TURN ? TA_WAVE : 1];
    const int b = blockIdx.y, tid = threadIdx.x, c = tid % LPR, slot = tid / LPR;
    const int L = a.seq_lens[(int64_t)b * a.sl_s];
    const int half = a.R / 2;
    const int rows_tok = a.Hq + (QUANT ? 2 : 1) * a.Hkv;
    const bool live = 16 * c < a.D;
    // columns of the lane's two runs in a rotated row, and in one that is taken as it is
    const bool turned = TURN && c < a.R / 16;
    const int t_c0 = turned ? 8 * c : a.R + 8 * (c - a.R / 16), t_c1 = t_c0 + (turned ? half : (a.D - a.R) / 2);
    const int v_c0 = 8 * c, v_c1 = 8 * c + a.D / 2;
    const int groups = (a.T + a.tokens - 1) / a.tokens;
    const float freq0 = TURN ? a.freqs[tid % half] : 0.f;  // of this thread's first entry of the table
    bool bad = false;
    for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
        const int t0 = grp * a.tokens, n = min(a.tokens, a.T - t0);
        uint4 raw[ROWS_AHEAD][2][V];
        // a block of heads: as many as the workgroup has rows at a time, and the last one of fewer takes several tokens at a time
        int m = min(RPP, rows_tok), tpp = RPP / m, tok0 = slot / m;
        RowsHead row = rows_head<BF16, QUANT>(a, b, slot - tok0 * m);
        bool as_is = !TURN || row.kind == 2;
        int c0 = as_is ? v_c0 : t_c0, c1 = as_is ? v_c1 : t_c1;
        auto fetch = [&](int tok) {
#pragma unroll
            for (int u = 0; u < ROWS_AHEAD; ++u)
                if (live && tok + u * tpp < n) {
                    const char *src = row.src + (t0 + tok + u * tpp) * row.src_st;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        raw[u][0][v] = *(const uint4 *)(src + c0 * ES + 16 * v);
                        raw[u][1][v] = *(const uint4 *)(src + c1 * ES + 16 * v);
                    }
                }
        };
        if (tok0 < tpp)
            fetch(tok0);                                   // (on its way while the length and the tree arrive)
        if (grp == (int)blockIdx.x) {
            bool bad_tree = false;
            if (TURN && a.parent) {
                const int depth = rows_depth(a, b, tid & 63, bad_tree);
                if (tid < TA_WAVE)
                    depths[tid] = depth;
            }
            const bool bad_len = L < 0 || (QUANT && (int64_t)L + a.T > (int64_t)a.capacity);
            bad = bad_len || bad_tree;
            if (bad && tid == 0 && blockIdx.x == 0) {
                const int bits = (bad_len ? TA_STATUS_BAD_SEQLEN : 0) | (bad_tree ? TA_STATUS_BAD_PARENT : 0);
                atomicOr(a.status, bits);
                if (a.status2)
                    atomicOr(a.status2, bits);
            }
            if (bad && !TURN)
                return;
        }
        __syncthreads();                                   // the tables of the group before are no longer read
        if (TURN && !bad)
            for (int k = tid; k < n * half; k += ROWS_THREADS) {
                const int i = k / half, j = k - i * half;
                const int d = a.parent ? depths[t0 + i] : t0 + i;
                turn[i][j] = rows_turn((double)L + (double)d, k == tid ? freq0 : a.freqs[j], a.amplitude);
            }
        if (QUANT && !bad && tid < n) {
            place[tid] = rows_place(a, b, L + t0 + tid);
            if (place[tid].page < 0) {
                atomicOr(a.status, TA_STATUS_BAD_PAGE);
                if (a.status2)
                    atomicOr(a.status2, TA_STATUS_BAD_PAGE);
            }
        }
        __syncthreads();
        for (int y0 = 0; y0 < rows_tok; y0 += RPP) {
            if (y0 > 0) {
                m = min(RPP, rows_tok - y0);
                tpp = RPP / m;
                tok0 = slot / m;
                row = rows_head<BF16, QUANT>(a, b, y0 + slot - tok0 * m);
                as_is = !TURN || row.kind == 2;
                c0 = as_is ? v_c0 : t_c0;
                c1 = as_is ? v_c1 : t_c1;
            }
            for (int tok1 = tok0; tok1 < n && tok0 < tpp; tok1 += ROWS_AHEAD * tpp) {
                if (y0 > 0 || tok1 > tok0)
                    fetch(tok1);
#pragma unroll
                for (int u = 0; u < ROWS_AHEAD; ++u) {
                    const int tok = tok1 + u * tpp;
                    if (tok >= n)
                        break;
                    // the row's columns: fp32 values where they are turned or are fp32, pairs of bf16 where those are enough
                    float e[2][8];
                    uint32_t pair[2][4];
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            const uint32_t w[4] = {raw[u][r][v].x, raw[u][r][v].y, raw[u][r][v].z, raw[u][r][v].w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (BF16) {
                                    pair[r][i] = live ? w[i] : 0u;
                                    e[r][2 * i] = __uint_as_float(pair[r][i] << 16);
                                    e[r][2 * i + 1] = __uint_as_float(pair[r][i] & 0xffff0000u);
                                } else {
                                    e[r][4 * v + i] = live ? __uint_as_float(w[i]) : 0.f;
                                }
                            }
                        }
                    if (TURN && turned && !as_is && !bad) {
                        if (TURN == ROWS_HALVES) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                rows_rotate(e[0][i], e[1][i], turn[tok][c0 + i]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                rows_rotate(e[0][2 * i], e[0][2 * i + 1], turn[tok][c0 / 2 + i]);
                                rows_rotate(e[1][2 * i], e[1][2 * i + 1], turn[tok][c1 / 2 + i]);
                            }
                        }
                        if (BF16) {
#pragma unroll
                            for (int r = 0; r < 2; ++r)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    pair[r][i] = q8_pack_bf16(e[r][2 * i], e[r][2 * i + 1]);
                        }
                    }
                    if (TURN && (row.kind == 0 || !QUANT) && live) {
                        char *dst = row.dense + (t0 + tok) * row.dense_st;
                        if (BF16) {
                            const uint4 nan = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
                            *(uint4 *)(dst + 2 * c0) = bad ? nan : make_uint4(pair[0][0], pair[0][1], pair[0][2], pair[0][3]);
                            *(uint4 *)(dst + 2 * c1) = bad ? nan : make_uint4(pair[1][0], pair[1][1], pair[1][2], pair[1][3]);
                        } else {
                            const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                *(float4 *)(dst + 4 * c0 + 16 * v) = bad ? make_float4(nan, nan, nan, nan)
                                    : make_float4(e[0][4 * v], e[0][4 * v + 1], e[0][4 * v + 2], e[0][4 * v + 3]);
                                *(float4 *)(dst + 4 * c1 + 16 * v) = bad ? make_float4(nan, nan, nan, nan)
                                    : make_float4(e[1][4 * v], e[1][4 * v + 1], e[1][4 * v + 2], e[1][4 * v + 3]);
                            }
                        }
                    }
                    if (QUANT && row.kind != 0) {              // (all lanes of a row are in here or none)
                        // the largest magnitude, as bits, which order as the values do; two bf16 at a time
                        auto over_row = [&](uint32_t top) {
#pragma unroll
                            for (int off = LPR / 2; off > 0; off >>= 1)
                                top = max(top, (uint32_t)__shfl_xor((int)top, off, TA_WAVE));
                            return top;
                        };
                        uint32_t top = 0;
                        if (BF16) {
                            q8_u16x2 m = {0, 0};
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                m = __builtin_elementwise_max(m, __builtin_bit_cast(q8_u16x2, pair[i / 4][i % 4] & 0x7fff7fffu));
                            top = (uint32_t)max(m.x, m.y) << 16;
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                top = max(top, __float_as_uint(e[i / 8][i % 8]) & 0x7fffffffu);
                        }
                        top = over_row(top);
                        if (top >= 0x7f800000u) {              // no number among them: the largest of the others
                            top = 0;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                if (BF16)
                                    top = max(top, max(q8_finite_bits(__uint_as_float(pair[i / 4][i % 4] << 16)),
                                                       q8_finite_bits(__uint_as_float(pair[i / 4][i % 4] & 0xffff0000u))));
                                else
                                    top = max(top, max(q8_finite_bits(e[i / 4][2 * (i % 4)]), q8_finite_bits(e[i / 4][2 * (i % 4) + 1])));
                            }
                            top = over_row(top);
                        }
                        if (!bad && place[tok].page >= 0) {
                            const RowsPlace at = place[tok];
                            const uint32_t byte = q8_scale_byte(top);
                            const float power = q8_power(byte);
                            char *dst = row.codes + at.page * row.code_sp + at.slot * row.code_ss;
                            if (live) {
#pragma unroll
                                for (int r = 0; r < 2; ++r)
                                    *(uint2 *)(dst + (r ? c1 : c0)) =
                                        BF16 ? make_uint2(q8_codes4(pair[r][0], pair[r][1], power), q8_codes4(pair[r][2], pair[r][3], power))
                                             : make_uint2(q8_codes4(e[r][0], e[r][1], e[r][2], e[r][3], power),
                                                          q8_codes4(e[r][4], e[r][5], e[r][6], e[r][7], power));
                            }
                            if (c == 0)
                                row.scale[at.page * row.scale_sp + at.slot * row.scale_ss] = (uint8_t)byte;
                        }
                    }
                }
            }
        }
    }
}

// The same for any head dimension, rotated part and alignment: a wave takes a row, a lane two pairs of columns and four others.
template <bool BF16, bool TURN, bool QUANT>
__global__ __launch_bounds__(ROWS_THREADS) void ta_rows_any_kernel(TARows a)
{
    constexpr int P = TA_MAX_HEAD_DIM / 2 / TA_WAVE, N = TA_MAX_HEAD_DIM / TA_WAVE;
    const int b = blockIdx.y, lane = threadIdx.x % TA_WAVE, wave = threadIdx.x / TA_WAVE;
    const int L = a.seq_lens[(int64_t)b * a.sl_s];
    const int half = TURN ? a.R / 2 : 0, rest = a.D - 2 * half;
    const int rows_tok = a.Hq + (QUANT ? 2 : 1) * a.Hkv;
    int depth = 0;
    bool bad_tree = false;
    if (TURN && a.parent)
        depth = rows_depth(a, b, lane, bad_tree);
    const bool bad_len = L < 0 || (QUANT && (int64_t)L + a.T > (int64_t)a.capacity);
    const bool bad = bad_len || bad_tree;
    if (bad && threadIdx.x == 0 && blockIdx.x == 0) {
        const int bits = (bad_len ? TA_STATUS_BAD_SEQLEN : 0) | (bad_tree ? TA_STATUS_BAD_PARENT : 0);
        atomicOr(a.status, bits);
        if (a.status2)
            atomicOr(a.status2, bits);
    }
    if (bad && !TURN)
        return;
    auto load = [](const void *src, int col) {
        return BF16 ? ta_bf16_to_f32(((const uint16_t *)src)[col]) : ((const float *)src)[col];
    };
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int d = a.parent ? __shfl(depth, t & 63, TA_WAVE) : t;
        RowsPlace at = {-1, 0};
        if (QUANT && !bad) {
            at = rows_place(a, b, L + t);
            if (at.page < 0 && threadIdx.x == 0) {
                atomicOr(a.status, TA_STATUS_BAD_PAGE);
                if (a.status2)
                    atomicOr(a.status2, TA_STATUS_BAD_PAGE);
            }
        }
        float2 cs[P];
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (TURN && lane + k * TA_WAVE < half)
                cs[k] = rows_turn((double)L + (double)d, a.freqs[lane + k * TA_WAVE], a.amplitude);
        for (int x = wave; x < rows_tok; x += ROWS_THREADS / TA_WAVE) {
            const RowsHead row = rows_head<BF16, QUANT>(a, b, x);
            const char *src = row.src + t * row.src_st;
            // values: no pairs, all columns are others
            const bool pairs = TURN && row.kind != 2;
            const int h = pairs ? half : 0, r0 = 2 * h, nr = pairs ? rest : a.D;
            float e[2 * P + N];
            int col[2 * P + N];
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int j = lane + k * TA_WAVE;
                const bool is = j < h;
                col[2 * k] = is ? (a.interleaved ? 2 * j : j) : -1;
                col[2 * k + 1] = is ? (a.interleaved ? 2 * j + 1 : j + half) : -1;
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                col[2 * P + k] = lane + k * TA_WAVE < nr ? r0 + lane + k * TA_WAVE : -1;
#pragma unroll
            for (int k = 0; k < 2 * P + N; ++k)
                e[k] = col[k] >= 0 ? load(src, col[k]) : 0.f;
            if (pairs) {
#pragma unroll
                for (int k = 0; k < P; ++k)
                    if (col[2 * k] >= 0)
                        rows_rotate(e[2 * k], e[2 * k + 1], cs[k]);
            }
            if (TURN && (row.kind == 0 || !QUANT)) {
                char *dst = row.dense + t * row.dense_st;
#pragma unroll
                for (int k = 0; k < 2 * P + N; ++k)
                    if (col[k] >= 0) {
                        if (BF16)
                            ((uint16_t *)dst)[col[k]] = bad ? (uint16_t)0x7fc0u : (uint16_t)(q8_pack_bf16(e[k], 0.f) & 0xffffu);
                        else
                            ((float *)dst)[col[k]] = bad ? __uint_as_float(0x7fc00000u) : e[k];
                    }
            }
            if (QUANT && row.kind != 0 && at.page >= 0) {
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 2 * P + N; ++k) {
                    if (TURN && BF16)
                        e[k] = __uint_as_float(q8_pack_bf16(e[k], 0.f) << 16);
                    top = max(top, q8_finite_bits(e[k]));
                }
                for (int off = TA_WAVE / 2; off > 0; off >>= 1)
                    top = max(top, (uint32_t)__shfl_xor((int)top, off, TA_WAVE));
                const uint32_t byte = q8_scale_byte(top);
                char *dst = row.codes + at.page * row.code_sp + at.slot * row.code_ss;
#pragma unroll
                for (int k = 0; k < 2 * P + N; ++k)
                    if (col[k] >= 0)
                        ((uint8_t *)dst)[col[k]] = (uint8_t)q8_codes4(e[k], 0.f, 0.f, 0.f, q8_power(byte));
                if (lane == 0)
                    row.scale[at.page * row.scale_sp + at.slot * row.scale_ss] = (uint8_t)byte;
            }
        }
    }
}

template <bool BF16, int TURN, bool QUANT>
static hipError_t launch_rows(const TARows &r, hipStream_t stream)
{
    const int tokens = r.vec ? r.tokens : 1, groups = (r.T + tokens - 1) / tokens;
    if (tokens < 1 || tokens > ROWS_TOKENS || r.R > TA_MAX_HEAD_DIM || r.D > TA_MAX_HEAD_DIM)
        return hipErrorInvalidValue;
    const dim3 grid(groups < 65536 ? groups : 65536, r.B), block(ROWS_THREADS);
    if (!r.vec)
        hipLaunchKernelGGL((ta_rows_any_kernel<BF16, TURN != ROWS_KEEP, QUANT>), grid, block, 0, stream, r);
    else if (r.D <= 16 * 4)
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 4>), grid, block, 0, stream, r);
    else if (r.D <= 16 * 8)
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 8>), grid, block, 0, stream, r);
    else
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 16>), grid, block, 0, stream, r);
    return hipGetLastError();
}

template <bool BF16>
static hipError_t launch_rows(const TARows &r, hipStream_t stream)
{
    const bool turn = r.freqs != nullptr, quant = r.k_out == nullptr && r.kc != nullptr;
    if (turn && quant)
        return r.interleaved ? launch_rows<BF16, ROWS_NEIGHBOURS, true>(r, stream) : launch_rows<BF16, ROWS_HALVES, true>(r, stream);
    if (turn)
        return r.interleaved ? launch_rows<BF16, ROWS_NEIGHBOURS, false>(r, stream) : launch_rows<BF16, ROWS_HALVES, false>(r, stream);
    return launch_rows<BF16, ROWS_KEEP, true>(r, stream);
}

hipError_t ta_launch_rows(const TARows &r, hipStream_t stream)
{
    return r.is_bf16 ? launch_rows<true>(r, stream) : launch_rows<false>(r, stream);
}

// Rows of the cache as dense ones.  The LPR lanes of a row take as many codes each as fill 16 bytes of output (PER; or one code,
// where rows do not start on 16 bytes), so that a row is written as one piece of memory.  What bounds it: the writes; a thread
// requests READ_AHEAD pieces before it writes the first (16 contexts of 1000 to 9000 tokens, 8 KV heads: 105 us, 4.7 TB/s
// read and written; one after the other 117).
constexpr int READ_AHEAD = 8, READ_TOKENS = 32;

template <bool BF16, int PER, int LPR>
__global__ __launch_bounds__(ROWS_THREADS) void ta_q8_read_kernel(TAQ8Read a)
{
    constexpr int ES = BF16 ? 2 : 4, RPP = ROWS_THREADS / LPR;
    __shared__ RowsPlace place[READ_TOKENS];
    const int b = blockIdx.y, c = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int start = a.starts ? a.starts[(int64_t)b * a.st_s] : 0, count = a.counts[(int64_t)b * a.ct_s];
    const bool bad = start < 0 || count < 0 || count > a.N || (int64_t)start + count > (int64_t)a.capacity;
    if (bad && threadIdx.x == 0 && blockIdx.x == 0)
        atomicOr(a.status, TA_STATUS_BAD_SEQLEN);
    const int end = bad ? a.N : count, groups = (end + a.tokens - 1) / a.tokens, rows_tok = 2 * a.Hkv;
    for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
        const int t0 = grp * a.tokens, n = min(a.tokens, end - t0);
        __syncthreads();                                   // the table of the group before is no longer read
        if ((int)threadIdx.x < n) {
            RowsPlace r = {b, start + t0 + (int)threadIdx.x};
            if (bad) {
                r.page = -1;
            } else if (a.page_table) {
                const int pos = start + t0 + (int)threadIdx.x, k = pos / a.ps;
                r.page = a.page_table[(int64_t)b * a.pt_sb + k];
                r.slot = pos - k * a.ps;
                if (r.page < 0 || r.page >= a.n_pages) {
                    r.page = -1;
                    atomicOr(a.status, TA_STATUS_BAD_PAGE);
                }
            }
            place[threadIdx.x] = r;
        }
        __syncthreads();
        // (heads and tokens as in ta_rows_kernel)
        for (int y0 = 0; y0 < rows_tok; y0 += RPP) {
            const int m = min(RPP, rows_tok - y0), tpp = RPP / m, tok0 = slot / m, y = y0 + slot - tok0 * m;
            const bool is_v = y >= a.Hkv;
            const int64_t h = is_v ? y - a.Hkv : y;
            const char *src = is_v ? (const char *)a.vc + h * a.v_sh : (const char *)a.kc + h * a.k_sh;
            const uint8_t *ssrc = is_v ? a.vs + h * a.vs_sh : a.ks + h * a.ks_sh;
            char *dst = is_v ? (char *)a.v_out + (b * a.vo_sb + t0 * a.vo_st + h * a.vo_sh) * ES
                             : (char *)a.k_out + (b * a.ko_sb + t0 * a.ko_st + h * a.ko_sh) * ES;
            const int64_t sp = is_v ? a.v_sp : a.k_sp, ss = is_v ? a.v_ss : a.k_ss, ssp = is_v ? a.vs_sp : a.ks_sp,
                          sss = is_v ? a.vs_ss : a.ks_ss, dst_st = (is_v ? a.vo_st : a.ko_st) * ES;
            for (int c0 = c * PER; c0 < a.D && tok0 < tpp; c0 += LPR * PER)            // (once, but for single codes)
                for (int tok1 = tok0; tok1 < n; tok1 += READ_AHEAD * tpp) {
                    uint32_t w[READ_AHEAD][2], sb[READ_AHEAD];
#pragma unroll
                    for (int u = 0; u < READ_AHEAD; ++u) {
                        const int tok = tok1 + u * tpp;
                        w[u][0] = w[u][1] = 0u;
                        sb[u] = 255u;
                        if (tok < n && place[tok].page >= 0) {
                            const RowsPlace at = place[tok];
                            const char *from = src + at.page * sp + at.slot * ss + c0;
                            sb[u] = ssrc[at.page * ssp + at.slot * sss];
                            if (PER == 8) {
                                const uint2 v = *(const uint2 *)from;
                                w[u][0] = v.x;
                                w[u][1] = v.y;
                            } else {
                                w[u][0] = PER == 4 ? *(const uint32_t *)from : (uint32_t) * (const uint8_t *)from;
                            }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < READ_AHEAD; ++u) {
                        const int tok = tok1 + u * tpp;
                        if (tok >= n)
                            break;
                        char *to = dst + tok * dst_st + c0 * ES;
                        const float scale = q8_scale(sb[u]);
                        float v[4];
                        if (PER != 8)
                            q8_values4(w[u][0], v);
                        if (PER == 8)
                            *(uint4 *)to = make_uint4(q8_bf16_2<false>(w[u][0], scale), q8_bf16_2<true>(w[u][0], scale),
                                                      q8_bf16_2<false>(w[u][1], scale), q8_bf16_2<true>(w[u][1], scale));
                        else if (PER == 4)
                            *(float4 *)to = make_float4(v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
                        else if (BF16)
                            *(uint16_t *)to = (uint16_t)(q8_pack_bf16(v[0] * scale, 0.f) & 0xffffu);
                        else
                            *(float *)to = v[0] * scale;
                    }
                }
        }
    }
}

template <bool BF16>
static hipError_t launch_read(const TAQ8Read &r, hipStream_t stream)
{
    constexpr int PER = BF16 ? 8 : 4;
    if (r.tokens < 1 || r.tokens > READ_TOKENS)
        return hipErrorInvalidValue;
    const int groups = (r.N + r.tokens - 1) / r.tokens;
    const dim3 grid(groups < 65536 ? groups : 65536, r.B), block(ROWS_THREADS);
    if (!r.vec)
        hipLaunchKernelGGL((ta_q8_read_kernel<BF16, 1, TA_WAVE>), grid, block, 0, stream, r);
    else if (r.D <= 64)
        hipLaunchKernelGGL((ta_q8_read_kernel<BF16, PER, 64 / PER>), grid, block, 0, stream, r);
    else if (r.D <= 128)
        hipLaunchKernelGGL((ta_q8_read_kernel<BF16, PER, 128 / PER>), grid, block, 0, stream, r);
    else
        hipLaunchKernelGGL((ta_q8_read_kernel<BF16, PER, 256 / PER>), grid, block, 0, stream, r);
    return hipGetLastError();
}

hipError_t ta_launch_q8_read(const TAQ8Read &r, hipStream_t stream)
{
    return r.is_bf16 ? launch_read<true>(r, stream) : launch_read<false>(r, stream);
}

// Bookkeeping after acceptance (see ta_compact_kernel): one workgroup per request; codes in pieces of type P, scales byte by byte.
// A phase reads every piece of some columns before it writes any of them, and no two phases touch the same bytes.
constexpr int Q8C_THREADS = 512, Q8C_REGS = 8;

template <typename P>
__global__ __launch_bounds__(Q8C_THREADS) void ta_q8_compact_kernel(TAQ8Compact c)
{
    __shared__ int ids[TA_MAX_TREE];
    __shared__ int64_t pages[TA_MAX_TREE], slots[TA_MAX_TREE];
    __shared__ int bad;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int L = c.seq_lens[(int64_t)b * c.sl_s];
    const int n = c.n_accepted[(int64_t)b * c.na_s];
    const bool n_ok = n >= 0 && n <= c.A;
    // the positions rows come from (L .. L+T-1) and go to (L .. L+n-1; a path may name a node twice and be longer than T)
    const int span = n_ok ? max(c.T, n) : c.T;
    const bool len_ok = L >= 0 && (int64_t)L + span <= (int64_t)c.capacity;
    const bool has_id = n_ok && tid < n, has_pos = len_ok && tid < span;
    int id = 0;
    int64_t page = b, slot = (int64_t)L + tid;
    if (has_id)
        id = c.accepted[(int64_t)b * c.acc_sb + tid];
    if (has_pos && c.page_table) {
        page = c.page_table[(int64_t)b * c.pt_sb + (L + tid) / c.ps];
        slot = (L + tid) % c.ps;
    }
    if (tid == 0)
        bad = 0;
    __syncthreads();
    if (has_id) {
        ids[tid] = id;
        if (id < 0 || id >= c.T)
            atomicOr(&bad, 1);
    }
    if (has_pos) {
        if (c.page_table && (page < 0 || page >= c.n_pages)) {     // a page the cache does not have
            atomicOr(&bad, 2);
            page = 0;
        }
        pages[tid] = page;
        slots[tid] = slot;
    }
    __syncthreads();
    const bool path_ok = n_ok && (bad & 1) == 0;
    const bool pages_ok = (bad & 2) == 0;
    if (!len_ok || !path_ok || !pages_ok) {
        if (tid == 0) {
            atomicOr(c.status, !len_ok ? TA_STATUS_BAD_SEQLEN : !path_ok ? TA_STATUS_BAD_PATH : TA_STATUS_BAD_PAGE);
            if (c.seq_lens_out)
                c.seq_lens_out[(int64_t)b * c.slo_s] = L;
        }
        return;
    }
    if (n > 0) {
        const int per_row = c.D / (int)sizeof(P);                  // pieces of a row
        auto move = [&](auto zero, int cols, auto piece) {         // (zero: a value of the pieces' type)
            typedef decltype(zero) Q;
            const int per_phase = Q8C_THREADS * Q8C_REGS / n;      // n <= TA_MAX_TREE: at least 64
            for (int c0 = 0; c0 < cols; c0 += per_phase) {
                const int nc = min(per_phase, cols - c0);
                Q r[Q8C_REGS];
#pragma unroll
                for (int k = 0; k < Q8C_REGS; ++k) {
                    const int x = tid + k * Q8C_THREADS;
                    if (x < nc * n)
                        r[k] = *piece(c0 + x % nc, ids[x / nc]);
                }
                __syncthreads();
#pragma unroll
                for (int k = 0; k < Q8C_REGS; ++k) {
                    const int x = tid + k * Q8C_THREADS;
                    if (x < nc * n)
                        *piece(c0 + x % nc, x / nc) = r[k];
                }
            }
        };
        move(P{}, 2 * c.Hkv * per_row, [&](int col, int tok) {
            const int u = col / per_row, g = u >> 1;
            char *base = (u & 1) ? (char *)c.v + pages[tok] * c.v_sp + slots[tok] * c.v_ss + (int64_t)g * c.v_sh
                                 : (char *)c.k + pages[tok] * c.k_sp + slots[tok] * c.k_ss + (int64_t)g * c.k_sh;
            return (P *)base + (col - u * per_row);
        });
        move(uint8_t{}, 2 * c.Hkv, [&](int col, int tok) {
            const int g = col >> 1;
            return (col & 1) ? c.vs + pages[tok] * c.vs_sp + (int64_t)g * c.vs_sh + slots[tok] * c.vs_ss
                             : c.ks + pages[tok] * c.ks_sp + (int64_t)g * c.ks_sh + slots[tok] * c.ks_ss;
        });
    }
    if (tid == 0 && c.seq_lens_out)
        c.seq_lens_out[(int64_t)b * c.slo_s] = L + n;
}

hipError_t ta_launch_q8_compact(const TAQ8Compact &c, hipStream_t stream)
{
    if (c.vec)
        hipLaunchKernelGGL(ta_q8_compact_kernel<uint4>, dim3(c.B), dim3(Q8C_THREADS), 0, stream, c);
    else
        hipLaunchKernelGGL(ta_q8_compact_kernel<uint8_t>, dim3(c.B), dim3(Q8C_THREADS), 0, stream, c);
    return hipGetLastError();
}
