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

// The row x of token t: where it comes from and what it is.
struct RowsRow {
    const void *src;
    int h;
    int kind;                               // 0 query, 1 key, 2 value
};

template <bool BF16>
__device__ __forceinline__ RowsRow rows_row(const TARows &a, int b, int t, int x)
{
    constexpr int ES = BF16 ? 2 : 4;
    RowsRow r;
    r.kind = x < a.Hq ? 0 : x < a.Hq + a.Hkv ? 1 : 2;
    r.h = r.kind == 0 ? x : r.kind == 1 ? x - a.Hq : x - a.Hq - a.Hkv;
    const char *base = (const char *)(r.kind == 0 ? a.q : r.kind == 1 ? a.k : a.v);
    const int64_t sb = r.kind == 0 ? a.q_sb : r.kind == 1 ? a.k_sb : a.v_sb, st = r.kind == 0 ? a.q_st : r.kind == 1 ? a.k_st : a.v_st,
                  sh = r.kind == 0 ? a.q_sh : r.kind == 1 ? a.k_sh : a.v_sh;
    r.src = base + ((int64_t)b * sb + (int64_t)t * st + (int64_t)r.h * sh) * ES;
    return r;
}

template <bool BF16>
__device__ __forceinline__ char *rows_dense(const TARows &a, int b, int t, const RowsRow &r)
{
    constexpr int ES = BF16 ? 2 : 4;
    return r.kind == 0 ? (char *)a.q_out + ((int64_t)b * a.qo_sb + (int64_t)t * a.qo_st + (int64_t)r.h * a.qo_sh) * ES
                       : (char *)a.k_out + ((int64_t)b * a.ko_sb + (int64_t)t * a.ko_st + (int64_t)r.h * a.ko_sh) * ES;
}

__device__ __forceinline__ char *rows_codes(const TARows &a, const RowsPlace &at, const RowsRow &r)
{
    return r.kind == 1 ? (char *)a.kc + at.page * a.k_sp + (int64_t)r.h * a.k_shc + at.slot * a.k_ss
                       : (char *)a.vc + at.page * a.v_sp + (int64_t)r.h * a.v_shc + at.slot * a.v_ss;
}

__device__ __forceinline__ uint8_t *rows_scale(const TARows &a, const RowsPlace &at, const RowsRow &r)
{
    return r.kind == 1 ? a.ks + at.page * a.ks_sp + (int64_t)r.h * a.ks_sh + at.slot * a.ks_ss
                       : a.vs + at.page * a.vs_sp + (int64_t)r.h * a.vs_sh + at.slot * a.vs_ss;
}

// Rotated (TURN) queries and keys to dense rows, or keys (rotated or not) and values into the cache (QUANT).  A lane holds sixteen
// columns of a row in two runs of eight, which are each other's partners where columns are paired across the halves, and
// neighbours otherwise; the LPR lanes of a row find its maximum among themselves.
template <bool BF16, bool TURN, bool QUANT, int LPR>
__global__ __launch_bounds__(ROWS_THREADS) void ta_rows_kernel(TARows a)
{
    constexpr int V = BF16 ? 1 : 2;                        // 16-byte loads of eight columns
    __shared__ float2 turn[TURN ? ROWS_TOKENS : 1][TURN ? TA_MAX_HEAD_DIM / 2 : 1];
    __shared__ RowsPlace place[ROWS_TOKENS];
    __shared__ int depths[TURN ? TA_WAVE : 1];
    const int b = blockIdx.y, tid = threadIdx.x, c = tid % LPR;
    const int L = a.seq_lens[(int64_t)b * a.sl_s];
    const int half = a.R / 2;
    const int rows_tok = a.Hq + (QUANT ? 2 : 1) * a.Hkv;
    bool bad_tree = false;
    if (TURN && a.parent) {
        const int depth = rows_depth(a, b, tid & 63, bad_tree);
        if (tid < TA_WAVE)
            depths[tid] = depth;
    }
    const bool bad_len = L < 0 || (QUANT && (int64_t)L + a.T > (int64_t)a.capacity);
    const bool bad = bad_len || bad_tree;
    if (bad && tid == 0 && blockIdx.x == 0) {
        const int bits = (bad_len ? TA_STATUS_BAD_SEQLEN : 0) | (bad_tree ? TA_STATUS_BAD_PARENT : 0);
        atomicOr(a.status, bits);
        if (a.status2)
            atomicOr(a.status2, bits);
    }
    if (bad && !TURN)
        return;
    const int groups = (a.T + a.tokens - 1) / a.tokens;
    for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
        const int t0 = grp * a.tokens, n = min(a.tokens, a.T - t0), total = n * rows_tok;
        uint4 raw[2][V];
        RowsRow row;
        int tok = 0;
        // columns of the lane's two runs
        const bool turned_cols = TURN && c < a.R / 16;
        auto columns = [&](bool value, int &c0, int &c1) {
            const bool apart = turned_cols && !a.interleaved && !value;
            c0 = apart ? 8 * c : 16 * c;
            c1 = apart ? half + 8 * c : 16 * c + 8;
        };
        auto fetch = [&](int x) {
            tok = x / rows_tok;
            row = rows_row<BF16>(a, b, t0 + tok, x - tok * rows_tok);
            int c0, c1;
            columns(row.kind == 2, c0, c1);
            if (16 * c < a.D) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    raw[0][v] = *(const uint4 *)((const char *)row.src + c0 * (BF16 ? 2 : 4) + 16 * v);
                    raw[1][v] = *(const uint4 *)((const char *)row.src + c1 * (BF16 ? 2 : 4) + 16 * v);
                }
            }
        };
        int x = tid / LPR;
        if (x < total)
            fetch(x);
        __syncthreads();                                   // the tables of the group before are no longer read
        if (TURN && !bad)
            for (int k = tid; k < n * half; k += ROWS_THREADS) {
                const int i = k / half, j = k - i * half;
                const int d = a.parent ? depths[t0 + i] : t0 + i;
                turn[i][j] = rows_turn((double)L + (double)d, a.freqs[j], a.amplitude);
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
        for (; x < total; x += ROWS_THREADS / LPR) {
            if (x >= ROWS_THREADS / LPR)
                fetch(x);
            const bool live = 16 * c < a.D;
            float e[2][8];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const uint32_t w[4] = {raw[r][v].x, raw[r][v].y, raw[r][v].z, raw[r][v].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (BF16) {
                            e[r][2 * i] = live ? __uint_as_float(w[i] << 16) : 0.f;
                            e[r][2 * i + 1] = live ? __uint_as_float(w[i] & 0xffff0000u) : 0.f;
                        } else {
                            e[r][4 * v + i] = live ? __uint_as_float(w[i]) : 0.f;
                        }
                    }
                }
            int c0, c1;
            columns(row.kind == 2, c0, c1);
            if (TURN && turned_cols && row.kind != 2) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 t = bad ? make_float2(__uint_as_float(0x7fc00000u), 0.f) : turn[tok][8 * c + i];
                    // (the pair of frequency 8 c + i: columns i of both runs, or neighbours within one of them)
                    float &p0 = a.interleaved ? e[i / 4][(2 * i) % 8] : e[0][i], &p1 = a.interleaved ? e[i / 4][(2 * i) % 8 + 1] : e[1][i];
                    rows_rotate(p0, p1, t);
                }
            }
            uint32_t packed[2][4];                         // bf16 rows: what is stored, and what is quantised
            if (TURN && BF16) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        packed[r][i] = q8_pack_bf16(e[r][2 * i], e[r][2 * i + 1]);
                        if (bad)
                            packed[r][i] = 0x7fc07fc0u;
                        if (QUANT) {
                            e[r][2 * i] = __uint_as_float(packed[r][i] << 16);
                            e[r][2 * i + 1] = __uint_as_float(packed[r][i] & 0xffff0000u);
                        }
                    }
            }
            if (TURN && (row.kind == 0 || !QUANT)) {
                char *dst = rows_dense<BF16>(a, b, t0 + tok, row);
                if (live) {
                    if (BF16) {
                        *(uint4 *)(dst + 2 * c0) = make_uint4(packed[0][0], packed[0][1], packed[0][2], packed[0][3]);
                        *(uint4 *)(dst + 2 * c1) = make_uint4(packed[1][0], packed[1][1], packed[1][2], packed[1][3]);
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
            }
            if (QUANT) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    top = max(top, q8_finite_bits(e[i / 8][i % 8]));
                for (int off = LPR / 2; off > 0; off >>= 1)
                    top = max(top, (uint32_t)__shfl_xor((int)top, off, TA_WAVE));
                if (row.kind != 0 && !bad && place[tok].page >= 0) {
                    const RowsPlace at = place[tok];
                    const uint32_t byte = q8_scale_byte(top);
                    const float inv = q8_inverse(byte);
                    char *dst = rows_codes(a, at, row);
                    if (live) {
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            *(uint2 *)(dst + (r ? c1 : c0)) =
                                make_uint2(q8_codes4(e[r][0] * inv, e[r][1] * inv, e[r][2] * inv, e[r][3] * inv),
                                           q8_codes4(e[r][4] * inv, e[r][5] * inv, e[r][6] * inv, e[r][7] * inv));
                    }
                    if (c == 0)
                        *rows_scale(a, at, row) = (uint8_t)byte;
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
            const RowsRow row = rows_row<BF16>(a, b, t, x);
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
                e[k] = col[k] >= 0 ? load(row.src, col[k]) : 0.f;
            if (pairs) {
#pragma unroll
                for (int k = 0; k < P; ++k)
                    if (col[2 * k] >= 0)
                        rows_rotate(e[2 * k], e[2 * k + 1], cs[k]);
            }
            if (TURN && (row.kind == 0 || !QUANT)) {
                char *dst = rows_dense<BF16>(a, b, t, row);
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
                const float inv = q8_inverse(byte);
                char *dst = rows_codes(a, at, row);
#pragma unroll
                for (int k = 0; k < 2 * P + N; ++k)
                    if (col[k] >= 0)
                        ((uint8_t *)dst)[col[k]] = (uint8_t)q8_codes4(e[k] * inv, 0.f, 0.f, 0.f);
                if (lane == 0)
                    *rows_scale(a, at, row) = (uint8_t)byte;
            }
        }
    }
}

template <bool BF16, bool TURN, bool QUANT>
static hipError_t launch_rows(const TARows &r, hipStream_t stream)
{
    const int tokens = r.vec ? r.tokens : 1, groups = (r.T + tokens - 1) / tokens;
    if (tokens < 1 || tokens > ROWS_TOKENS || r.R > TA_MAX_HEAD_DIM || r.D > TA_MAX_HEAD_DIM)
        return hipErrorInvalidValue;
    const dim3 grid(groups < 65536 ? groups : 65536, r.B), block(ROWS_THREADS);
    if (!r.vec)
        hipLaunchKernelGGL((ta_rows_any_kernel<BF16, TURN, QUANT>), grid, block, 0, stream, r);
    else if (r.D <= 16 * 4)
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 4>), grid, block, 0, stream, r);
    else if (r.D <= 16 * 8)
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 8>), grid, block, 0, stream, r);
    else
        hipLaunchKernelGGL((ta_rows_kernel<BF16, TURN, QUANT, 16>), grid, block, 0, stream, r);
    return hipGetLastError();
}

hipError_t ta_launch_rows(const TARows &r, hipStream_t stream)
{
    const bool turn = r.freqs != nullptr, quant = r.k_out == nullptr && r.kc != nullptr;
    if (turn && quant)
        return r.is_bf16 ? launch_rows<true, true, true>(r, stream) : launch_rows<false, true, true>(r, stream);
    if (turn)
        return r.is_bf16 ? launch_rows<true, true, false>(r, stream) : launch_rows<false, true, false>(r, stream);
    return r.is_bf16 ? launch_rows<true, false, true>(r, stream) : launch_rows<false, false, true>(r, stream);
}

// Rows of the cache as dense ones.  A lane takes sixteen codes (or, VEC false, one).
template <bool BF16, bool VEC>
__global__ __launch_bounds__(ROWS_THREADS) void ta_q8_read_kernel(TAQ8Read a)
{
    constexpr int ES = BF16 ? 2 : 4, PER = VEC ? 16 : 1;
    const int b = blockIdx.y;
    const int start = a.starts ? a.starts[(int64_t)b * a.st_s] : 0, count = a.counts[(int64_t)b * a.ct_s];
    const bool bad = start < 0 || count < 0 || count > a.N || (int64_t)start + count > (int64_t)a.capacity;
    if (bad && threadIdx.x == 0 && blockIdx.x == 0)
        atomicOr(a.status, TA_STATUS_BAD_SEQLEN);
    const int end = bad ? a.N : count, groups = (end + a.tokens - 1) / a.tokens;
    const int lpr = (a.D + PER - 1) / PER, rows_tok = 2 * a.Hkv;
    for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
        const int t0 = grp * a.tokens, n = min(a.tokens, end - t0), total = n * rows_tok * lpr;
        for (int x = threadIdx.x; x < total; x += ROWS_THREADS) {
            const int r = x / lpr, c = x - r * lpr, tok = r / rows_tok, y = r - tok * rows_tok;
            const bool is_v = y >= a.Hkv;
            const int h = is_v ? y - a.Hkv : y, t = t0 + tok;
            int64_t page = b, slot = (int64_t)start + t;
            bool lost = bad;
            if (!bad && a.page_table) {
                const int pos = start + t, k = pos / a.ps;
                page = a.page_table[(int64_t)b * a.pt_sb + k];
                slot = pos - k * a.ps;
                if (page < 0 || page >= a.n_pages) {
                    lost = true;
                    if (y == 0 && c == 0)
                        atomicOr(a.status, TA_STATUS_BAD_PAGE);
                }
            }
            float scale = __uint_as_float(0x7fc00000u);
            uint32_t w[4] = {0u, 0u, 0u, 0u};
            if (!lost) {
                const char *src = is_v ? (const char *)a.vc + page * a.v_sp + (int64_t)h * a.v_sh + slot * a.v_ss
                                       : (const char *)a.kc + page * a.k_sp + (int64_t)h * a.k_sh + slot * a.k_ss;
                scale = q8_scale(is_v ? a.vs[page * a.vs_sp + (int64_t)h * a.vs_sh + slot * a.vs_ss]
                                      : a.ks[page * a.ks_sp + (int64_t)h * a.ks_sh + slot * a.ks_ss]);
                if (VEC) {
                    const uint4 u = *(const uint4 *)(src + 16 * c);
                    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
                } else {
                    w[0] = ((const uint8_t *)src)[c];
                }
            }
            char *dst = is_v ? (char *)a.v_out + ((int64_t)b * a.vo_sb + (int64_t)t * a.vo_st + (int64_t)h * a.vo_sh) * ES
                             : (char *)a.k_out + ((int64_t)b * a.ko_sb + (int64_t)t * a.ko_st + (int64_t)h * a.ko_sh) * ES;
            if (VEC) {
#pragma unroll
                for (int i = 0; i < 4; i += BF16 ? 2 : 1) {
                    float v[8];
                    q8_values4(w[i], v);
                    if (BF16) {
                        q8_values4(w[i + 1], v + 4);
                        *(uint4 *)(dst + 32 * c + 8 * i) =
                            make_uint4(q8_pack_bf16(v[0] * scale, v[1] * scale), q8_pack_bf16(v[2] * scale, v[3] * scale),
                                       q8_pack_bf16(v[4] * scale, v[5] * scale), q8_pack_bf16(v[6] * scale, v[7] * scale));
                    } else {
                        *(float4 *)(dst + 64 * c + 16 * i) = make_float4(v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
                    }
                }
            } else if (BF16) {
                ((uint16_t *)dst)[c] = (uint16_t)(q8_pack_bf16(q8_value(w[0]) * scale, 0.f) & 0xffffu);
            } else {
                ((float *)dst)[c] = q8_value(w[0]) * scale;
            }
        }
    }
}

hipError_t ta_launch_q8_read(const TAQ8Read &r, hipStream_t stream)
{
    const int groups = (r.N + r.tokens - 1) / r.tokens;
    const dim3 grid(groups < 65536 ? groups : 65536, r.B), block(ROWS_THREADS);
    if (r.vec && r.is_bf16)
        hipLaunchKernelGGL((ta_q8_read_kernel<true, true>), grid, block, 0, stream, r);
    else if (r.vec)
        hipLaunchKernelGGL((ta_q8_read_kernel<false, true>), grid, block, 0, stream, r);
    else if (r.is_bf16)
        hipLaunchKernelGGL((ta_q8_read_kernel<true, false>), grid, block, 0, stream, r);
    else
        hipLaunchKernelGGL((ta_q8_read_kernel<false, false>), grid, block, 0, stream, r);
    return hipGetLastError();
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
