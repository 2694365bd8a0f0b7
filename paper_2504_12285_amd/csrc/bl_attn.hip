/* Causal attention over the key/value cache of 8-bit codes (bitlinear.h, bl_attn_kv8).
 *
 * For one key/value head the rows of a request are its (query, head of the group) pairs: row r is query r / G, head r % G,
 * G = n_q / n_kv.  Per row the softmax runs over tiles of 64 tokens with a running reference m and a running sum:
 *     x_j = S_j * a + log2(vs)          S_j = <q pieces, codes of k_j>, a = softmax_scale * log2(e) * scale of q * ks
 *     w_j = 2^(x_j - m + 6)             the weight with the scale vs of its V block in it
 *     l  += w_j / vs,  O += w_j * codes of v_j,  out = O / l
 * with one ks and vs for the 16 tokens that share a block.  m moves only when a tile brings an x more than 8 above it
 * (weights then reach 2^14, inside fp16), so that most tiles rescale nothing and exchange nothing between lanes.
 *
 * S is computed transposed (tokens x rows), so that a lane holds the weights of ONE row for sixteen tokens, exactly what the
 * second product wants of it: the weights never leave the lane.  Which tokens a lane gets is chosen by the
 * order in which the rows of K are handed in, such that its V codes are consecutive in memory. */
#include <algorithm>
#include <type_traits>

#include "bl_device.h"
#include "bl_kv.h"

typedef _Float16 at_v8h __attribute__((ext_vector_type(8)));
typedef _Float16 at_v2h __attribute__((ext_vector_type(2)));
typedef float at_v16f __attribute__((ext_vector_type(16)));
typedef int at_v8i __attribute__((ext_vector_type(8)));
typedef uint32_t at_v4u __attribute__((ext_vector_type(4)));

#define AT_TILE 64                 /* tokens a tile */
#define AT_THREADS 256
#define AT_WAVES 4
/* Rows of a request and kv head up to which at_few does it: the columns of its products.  Fewer by at_many, measured, us, at_few against it: heads of 128, 8 to 16
 * rows, one request over 1000 tokens 10.4 to 11.8 against 16.5, over 8000 15.5 to 18.6 against 21, 64 over 4000 73 to 83 against 140; heads of 64, one over
 * 1000 6.8 against 13, 64 over 4000 45 against 106 to 121; the other way only one over 8000, heads of 64, 22 to 26 against 18. */
#define AT_FEW 16
#define AT_MANY 128                /* rows a workgroup of at_many */
#define AT_STREAM_GROUPS 512       /* workgroups of at_few: two a unit */
#define AT_STREAMS (AT_STREAM_GROUPS * AT_WAVES)
#define AT_GROW 8.0f
#define AT_LIFT 6.0f

struct at_args {
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    const uint16_t* q;
    const int* q_start;
    const int* seq_len;
    const int* table;
    uint16_t* out;
    float* part;                   /* workspace of at_few, and of at_many */
    float* many_part;
    uint32_t k_units, v_units;     /* 16-byte units from a block to the next */
    int64_t scale_stride, q_stride, out_stride, table_stride;
    int n_blocks, n_kv, G, n_q, B, T, shift, max_tokens, window;
    float factor;                  /* softmax_scale * log2(e) */
    int few_rows;                  /* rows of a request and kv head up to which at_few does it: AT_FEW, or 0 where it is not launched */
    int splits;                    /* of at_many */
    int part_skip;                 /* floats in front of the partial results of at_few: where each request's tiles end */
    /* of prefixes that requests share (bl_attn_kv8_shared) */
    const int* group;
    const int* shared_blocks;
    const int* shared_table;
    int64_t shared_stride;
    int2* pieces;                  /* [T] of each row: at_pieces, and at_query */
    float* part_ml;                /* reference and sum of each partial result */
    int64_t part_stride, own_at;   /* results a piece of a prefix or of at_few's has, and in front of those of at_many's own pieces */
    int n_groups, max_shared, group_splits, few_splits, many_splits, by_request;
    int apart;                     /* rows of a request and kv head from which it is no part of its group */
};

/* ---- what both kernels share --------------------------------------------------------------------------------------- */

__device__ __forceinline__ int at_uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float at_xor(float v, int m) { return __shfl_xor(v, m); }

/* A request: queries, tokens, and the tiles that its queries i0..i1 can see. */
struct at_request {
    int row0, n, len;
    int skip = 0;                  /* tokens in front that its group has */
};
__device__ __forceinline__ at_request at_read(const at_args& A, int b) {
    at_request r;
    const int a = A.q_start[b], e = A.q_start[b + 1];
    r.row0 = a < 0 ? 0 : a;
    const int end = e > A.T ? A.T : e;
    r.n = end > r.row0 ? end - r.row0 : 0;
    const int L = A.seq_len[b];
    r.len = L < 0 ? 0 : L > A.max_tokens ? A.max_tokens : L;
    return r;
}
/* Tokens of group g's prefix; 0 where there is no such group. */
__device__ __forceinline__ int at_shared_tokens(const at_args& A, int g) {
    if ((unsigned)g >= (unsigned)A.n_groups) return 0;
    const int s = A.shared_blocks[g];
    return (s < 0 ? 0 : s > A.max_shared ? A.max_shared : s) << A.shift;
}
__device__ __forceinline__ bool at_grouped(const at_args& A, int n) { return n * A.G < A.apart; }
template <bool SHARED>
__device__ __forceinline__ at_request at_read_own(const at_args& A, int b) {
    at_request r = at_read(A, b);
    if (SHARED) r.skip = at_shared_tokens(A, A.group[b]);
    return r;
}
/* First token that query i sees, and the one behind its last. */
__device__ __forceinline__ int at_from(const at_args& A, const at_request& r, int i) {
    const int p = A.window ? r.len - r.n + i - A.window + 1 : 0;
    return p > r.skip ? p : r.skip;
}
__device__ __forceinline__ int at_to(const at_request& r, int i) {
    const int e = r.len - r.n + i + 1;
    return e > 0 ? e : 0;
}

/* Sixteen codes of one feature (consecutive tokens) as fp16, exact. */
template <int KIND>
__device__ __forceinline__ void at_half16(bl_v4i c, at_v8h& lo, at_v8h& hi) {
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (KIND == BL_KV_INT8) {
            /* 0x6400 | u is 1024 + u in fp16; u = c + 128 */
            const uint32_t u = (uint32_t)c[i] ^ 0x80808080u;
            const at_v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
            o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(at_v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off);
            o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(at_v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off);
        } else {
            o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i], 1.0f, false));
            o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i], 1.0f, true));
        }
    }
    lo = __builtin_bit_cast(at_v8h, (at_v4u){o[0], o[1], o[2], o[3]});
    hi = __builtin_bit_cast(at_v8h, (at_v4u){o[4], o[5], o[6], o[7]});
}
/* The first n (0..16) codes of sixteen, zeros behind them. */
__device__ __forceinline__ bl_v4i at_first(bl_v4i c, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = n - 4 * i;
        c[i] = k >= 4 ? c[i] : k <= 0 ? 0 : c[i] & (int)((1u << (8 * k)) - 1);
    }
    return c;
}
__device__ __forceinline__ uint32_t at_pack_half(float a, float b) {
    const bl_v2f v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, at_v2h));
}

/* Sixteen bf16 values of q as the two 8-bit pieces that are multiplied with codes.
 * int8: t = rint(q * inv), |t| <= 127 * 256, t = 256 * hi + lo with lo in -128..127.
 * e4m3: t = q * inv, inv a power of two, hi = e4m3(t), lo = e4m3(t - hi): exact down to 2^-9 of the row's largest. */
template <int KIND>
__device__ __forceinline__ void at_pieces(const uint32_t (&w)[8], float inv, bl_v4i& hi, bl_v4i& lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = w[2 * i + (j >> 1)];
            t[j] = (j & 1 ? __uint_as_float(x & 0xffff0000u) : bl_bf16_to_f32(x & 0xffffu)) * inv;
        }
        if (KIND == BL_KV_INT8) {
            uint32_t a = 0, b = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = (int)rintf(t[j]), h = (v + 128) >> 8;
                a |= (uint32_t)(h & 0xff) << (8 * j);
                b |= (uint32_t)((v - 256 * h) & 0xff) << (8 * j);
            }
            hi[i] = (int)a, lo[i] = (int)b;
        } else {
            int a = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
            a = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], a, true);
            hi[i] = a;
            int b = __builtin_amdgcn_cvt_pk_fp8_f32(t[0] - __builtin_amdgcn_cvt_f32_fp8(a, 0), t[1] - __builtin_amdgcn_cvt_f32_fp8(a, 1), 0, false);
            b = __builtin_amdgcn_cvt_pk_fp8_f32(t[2] - __builtin_amdgcn_cvt_f32_fp8(a, 2), t[3] - __builtin_amdgcn_cvt_f32_fp8(a, 3), b, true);
            lo[i] = b;
        }
    }
}
/* Multiplier of a row of q, and the scale of what it gives, from its largest |q| (0: all zero).
 * A power of two that takes the largest to [2^(e-127), 2^(e-126)). */
__device__ __forceinline__ void at_power_scale(float most, int e, float& inv, float& scale) {
    e -= (int)(__float_as_uint(most) >> 23);
    e = e > 120 ? 120 : e < -120 ? -120 : e;
    inv = most > 0.0f ? __uint_as_float((uint32_t)(127 + e) << 23) : 0.0f;
    scale = __uint_as_float((uint32_t)(127 - e) << 23);
}
/* For at_pieces: 32512 / largest (int8), or to [128, 256). */
template <int KIND>
__device__ __forceinline__ void at_row_scale(float most, float& inv, float& scale) {
    if (KIND == BL_KV_INT8) {
        inv = most > 0.0f ? bl_div_rn(32512.0f, most) : 0.0f;
        scale = most * (1.0f / 32512.0f);
    } else {
        at_power_scale(most, 134, inv, scale);
    }
}
/* The largest |value| so far, and whether one is no finite number (such a row of q gives NaN, whatever its conversion makes of it). */
__device__ __forceinline__ float at_largest(const uint32_t (&w)[8], float most, bool& odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = (w[i] << 16) & 0x7fffffffu, b = w[i] & 0x7fff0000u;
        odd |= a >= 0x7f800000u || b >= 0x7f800000u;
        most = bl_max_pos(most, bl_max_pos(__uint_as_float(a), __uint_as_float(b)));
    }
    return most;
}

/* What is added to a score of a block whose V scale has the logarithm lv.  Where a row has seen nothing yet (m = -inf), or lv is
 * none, a masked score of -inf has to stay -inf: no infinity of the other sign is added. */
__device__ __forceinline__ float at_shift(float lv, float m) { return fminf(lv + AT_LIFT - m, 1e30f); }
/* Bytes from block 0 to block b, `units` of 16 bytes a block. */
__device__ __forceinline__ int64_t at_far(int b, uint32_t units) { return (int64_t)(((uint64_t)(uint32_t)b * units) << 4); }

/* Sum over the lanes up to this one: inside rows of 16, then across them. */
__device__ __forceinline__ int at_scan(int v) {
    v += bl_dpp<0x111>(v);                                  /* row_shr 1, 2, 4, 8 */
    v += bl_dpp<0x112>(v);
    v += bl_dpp<0x114>(v);
    v += bl_dpp<0x118>(v);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   /* row_bcast 15 into rows 1 and 3 */
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   /* row_bcast 31 into rows 2 and 3 */
    return v;
}
/* f(b) summed up to and with request b, for all of them, into s_upto; per thread consecutive requests.  s: AT_WAVES values. */
template <typename F>
__device__ __forceinline__ void at_sums(int B, F f, int* s_upto, int* s) {
    const int per = (B + AT_THREADS - 1) / AT_THREADS, tid = threadIdx.x;
    int mine = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < B) mine += f(tid * per + i);
    const int x = at_scan(mine);
    if ((tid & 63) == 63) s[tid >> 6] = x;
    __syncthreads();
    int sum = x - mine;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) sum += w < (tid >> 6) ? s[w] : 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < B) s_upto[tid * per + i] = sum += f(tid * per + i);
    __syncthreads();
}

/* ---- few rows: the cache is streamed ------------------------------------------------------------------------------ */

/* Tiles of request b in at_few, per kv head: one at least where it has rows to write, none where it is another's. */
__device__ __forceinline__ int at_few_tiles(const at_args& A, const at_request& r) {
    const int64_t rows = (int64_t)r.n * A.G;
    if (rows == 0 || rows > AT_FEW) return 0;
    const int t = (r.len + AT_TILE - 1) / AT_TILE - at_from(A, r, 0) / AT_TILE;
    return t > 0 ? t : 1;
}
/* Head h's rows of a request that brings more queries than the launch was made for (max_q), where none of its kernels does them: no numbers, so that
 * what the output held before passes for no result.  `threads` threads share them. */
template <int D>
__device__ __forceinline__ void at_no_rows(const at_args& A, const at_request& r, int h, int thread, int threads) {
    const int units = A.G * (D / 8);                         /* of 16 bytes */
    for (int64_t i = thread; i < (int64_t)r.n * units; i += threads)
        *bl_g((at_v4u*)(A.out + (r.row0 + i / units) * A.out_stride + (int64_t)h * A.G * D + i % units * 8)) = (at_v4u){0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
}
/* Tiles of a piece where `tiles` are split, and how many pieces have some. */
__device__ __forceinline__ int at_piece(int tiles, int splits) { return (tiles + splits - 1) / splits; }
__device__ __forceinline__ int at_piece_count(int tiles, int splits) {
    const int each = at_piece(tiles, splits);
    return each ? (tiles + each - 1) / each : 0;
}
/* A row's partial results: `prefix` of its group's prefix and `own` of its own tokens, whose sum is its output where there are any (0: it is done); many: the
 * own ones are at_many's.  AT_NO_NUMBERS: more queries than the launch was made for. */
#define AT_NO_NUMBERS -1
__device__ __forceinline__ int at_pieces(int prefix, int own, bool many) { return prefix | own << 8 | (many ? 1 << 16 : 0); }
/* Query i of request b, where partial results stand by requests, not by rows of the batch, because that is less: fewer than `apart` rows of each have some, however
 * many a prompt beside them brings (one of 8192 beside seven decoding requests: 0.1 GB for 3.9). */
__device__ __forceinline__ int at_query(const at_args& A, int b, int i) { return b * A.apart + i; }
/* Where the first piece of (row, head) stands among the partial results. */
__device__ __forceinline__ int64_t at_part_at(const at_args& A, int query, int row, int head) {
    if (!A.by_request) return (int64_t)row * A.n_q + head;
    return ((int64_t)(query / A.apart) * A.n_kv + head / A.G) * A.apart + query % A.apart * A.G + head % A.G;
}
/* Tiles a wave does, of `all` in the launch. */
__device__ __forceinline__ int at_share(int all) {
    const int s = (all + AT_STREAMS - 1) / AT_STREAMS;
    return s > 1 ? s : 1;
}
template <int D>
struct at_slot {                    /* a wave's partial result: rows x (D sums, m, l) */
    static constexpr int floats = AT_FEW * (D + 2);
};

/* The tiles of all requests and kv heads stand in one line (request, head, tile); a wave takes an equal piece of it, and a
 * piece may end one head's tiles and begin the next's.  What a piece has of an item that others share goes to the
 * workspace (at most two such: at its ends) and bl_attn_join adds it up.  The four pieces of a workgroup that lie in one item
 * (at_together) are taken tile by tile in turn instead, and meet in LDS: a quarter of the partial results.
 * ITEM (0, or the waves of a workgroup): a workgroup has one item whole, so that nothing is left to join (short contexts).
 * SHARED: a workgroup has one of `few_splits` pieces of what an item has behind its group's prefix, and leaves a partial result (as items, not in streams: what
 * a request has of its own is short, and a row's pieces are then known by its tiles alone).
 * ALONE: no at_many stands beside it; requests of more than AT_FEW rows then get no numbers (in the streams' form a lane's own work: an error's speed).
 * K rows of a tile go straight from memory into the registers that the matrix cores read (four 16 x 128 products of
 * codes against the two pieces of q), then V the same way.  V of a tile and K of the next are in flight while one computes,
 * and the block numbers of the one behind: also across the items of a piece.
 * Bound by the cache's stream: 64 requests over 8192 tokens, 241 MB, 46 us = 5.2 TB/s; two over 131071, 513 MB, 97 us = 5.3 (a read that
 * does nothing else 7.0; what is fetched is what the codes take).  About 5 us are the chain lengths -> blocks -> codes and
 * the last waves.  The codes' conversion and the softmax are 460 vector instructions a tile: a third of what its 16 KB allow. */
/* Whether workgroup g's four pieces, whole ones, lie in the item of tiles first .. last of the line. */
__device__ __forceinline__ bool at_together(int g, int share, int first, int last) {
    return (int64_t)g * AT_WAVES * share >= first && (int64_t)(g + 1) * AT_WAVES * share - 1 <= last;
}
template <int D, int WAVES>
struct at_meet_lds {                /* the waves' shares of one item */
    float o[WAVES][AT_FEW][D + 4], m[WAVES][AT_FEW], l[WAVES][AT_FEW];
};
template <int D>
struct at_few_lds {
    int upto[BL_KV_MAX_REQUESTS];
    int2 request[BL_KV_MAX_REQUESTS];                        /* first row * 32 + queries (31: 31 or more, not at_few's), tokens */
    int scan[AT_WAVES];
};
template <int D>
union at_stream_lds {
    at_few_lds<D> few;
    at_meet_lds<D, AT_WAVES> meet;
};
struct at_spot {
    int b, h, t, c, tile0;          /* request, kv head, tile of c, first tile */
};
template <int KIND, int D, bool WIDE, int ITEM, bool ALONE, bool SHARED = false>
__device__ __forceinline__ void at_few(const at_args& A, int group, uint8_t* lds_bytes) {
    constexpr int KS = D / 64, DT = D / 16, WAVES = ITEM ? ITEM : AT_WAVES;     /* 64-byte steps of a K row, 16-feature tiles of V */
    at_few_lds<D>& lds = *(at_few_lds<D>*)lds_bytes;
    const int tid = threadIdx.x, lane = tid & 63, wave = at_uniform(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    at_spot cur, next, after;                                /* the tile computed, the one loaded, the one whose blocks are read */
    int upto = 0, all = 0, share = 1, stream = group * AT_WAVES, count, begun0 = 0;
    bool together = true, small = true, alone = true;       /* the waves take one item's tiles in turn; have all of it */
    at_request mine = {0, 0, 0};
    auto upto_of = [&](int b) { return small ? __builtin_amdgcn_readlane(upto, b) : at_uniform(lds.upto[b]); };
    auto request = [&](int b) -> at_request {
        if (ITEM) return mine;
        if (small) return {__builtin_amdgcn_readlane(mine.row0, b), __builtin_amdgcn_readlane(mine.n, b), __builtin_amdgcn_readlane(mine.len, b)};
        const int2 r = lds.request[b];
        const int x = at_uniform(r.x);
        return {x >> 5, x & 31, at_uniform(r.y)};
    };
    /* the request that has tile `at` of the line (of one kv head) */
    auto find = [&](int at, at_spot& s) -> int {
        if (small) {
            s.b = __builtin_ctzll(__ballot(upto > at));
        } else {
            int lo = -1, hi = A.B - 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (lds.upto[mid] > at) hi = mid;
                else lo = mid;
            }
            s.b = at_uniform(hi);
        }
        const int before = s.b ? upto_of(s.b - 1) : 0;
        s.c = upto_of(s.b) - before, s.tile0 = at_from(A, request(s.b), 0) / AT_TILE;
        return before;
    };
    auto go_to = [&](int x) {
        const int before = find(x / A.n_kv, cur) * A.n_kv, r = x - before;
        cur.h = r / cur.c, cur.t = r % cur.c;
        return before + cur.h * cur.c;
    };
    int piece = 0;
    bool whole_item = !SHARED;
    if constexpr (ITEM) {
        if (SHARED) piece = group % A.few_splits, group /= A.few_splits;
        cur.b = group / A.n_kv, cur.h = group % A.n_kv;
        mine = at_read_own<SHARED>(A, cur.b);
        mine = {at_uniform(mine.row0), at_uniform(mine.n), at_uniform(mine.len), SHARED ? at_uniform(mine.skip) : 0};
        cur.c = at_few_tiles(A, mine), cur.t = wave;
        if (!cur.c) {
            if (SHARED) {
                if (ALONE && piece == 0 && cur.h == 0)
                    for (int i = tid; i < mine.n; i += AT_THREADS) A.pieces[mine.row0 + i] = make_int2(AT_NO_NUMBERS, 0);
            } else if (ALONE) {
                at_no_rows<D>(A, mine, cur.h, tid, WAVES * BL_WAVE);
            }
            return;
        }
        cur.tile0 = at_from(A, mine, 0) / AT_TILE;
        if (SHARED) {
            const int each = at_piece(cur.c, A.few_splits), all = cur.c, n = at_piece_count(all, A.few_splits);
            whole_item = mine.skip == 0 && n == 1;
            if (piece == 0 && cur.h == 0 && tid < mine.n)
                A.pieces[mine.row0 + tid] = make_int2(whole_item ? 0 : at_pieces(at_piece_count((mine.skip + AT_TILE - 1) / AT_TILE, A.group_splits), n, false), at_query(A, cur.b, tid));
            cur.tile0 += piece * each;
            cur.c = all - piece * each < each ? all - piece * each : each;
            if (cur.c <= 0) return;
        }
        count = (cur.c - wave + WAVES - 1) / WAVES;     /* (none for some waves of a short item: they bring nothing to the meeting) */
    } else {
        /* where each request's tiles end: up to 64 requests by every wave for itself, a lane each, more through LDS */
        small = A.B <= 64;
        int4* const heads = (int4*)A.part;                   /* bl_attn_join reads them there: tiles up to it, first row, queries */
        if (small) {
            if (lane < A.B) {
                mine = at_read(A, lane);
                upto = at_few_tiles(A, mine);
                if (ALONE && __builtin_expect(mine.n * A.G > AT_FEW, 0))
                    for (int h = group; h < A.n_kv; h += AT_STREAM_GROUPS) at_no_rows<D>(A, mine, h, wave, AT_WAVES);
            }
            upto = at_scan(upto);
            if (group == 0 && tid < A.B) heads[tid] = make_int4(upto, mine.row0, mine.n, 0);
        } else {
            at_sums(A.B, [&](int b) { return at_few_tiles(A, at_read(A, b)); }, lds.upto, lds.scan);
            for (int b = tid; b < A.B; b += AT_THREADS) {
                const at_request r = at_read(A, b);
                lds.request[b] = make_int2(r.row0 << 5 | (r.n < 31 ? r.n : 31), r.len);
                if (group == 0) heads[b] = make_int4(lds.upto[b], r.row0, r.n, 0);
                if (ALONE && __builtin_expect(r.n * A.G > AT_FEW, 0))
                    for (int h = group; h < A.n_kv; h += AT_STREAM_GROUPS) at_no_rows<D>(A, r, h, 0, 1);
            }
            __syncthreads();
        }
        all = upto_of(small ? 63 : A.B - 1) * A.n_kv, share = at_share(all);
        if ((int64_t)stream * share >= all) return;
        count = share;
        const int first = go_to(stream * share);
        together = at_together(group, share, first, first + cur.c - 1);
        begun0 = cur.t, alone = cur.c == share * AT_WAVES;
        if (together) {
            cur.t += wave;
        } else {
            stream += wave;
            const int64_t x0 = (int64_t)stream * share;
            if (x0 >= all) return;
            if (wave) go_to((int)x0);
            if (count > all - (int)x0) count = all - (int)x0;
        }
    }
    auto advance = [&](at_spot s) -> at_spot {
        if (ITEM || together) {
            s.t += WAVES;
        } else if (++s.t == s.c) {
            s.t = 0;
            if (++s.h == A.n_kv) {
                s.h = 0;
                find(upto_of(s.b), s);
            }
        }
        return s;
    };
    next = count > 1 ? advance(cur) : cur;
    after = count > 2 ? advance(next) : next;

    const int bs1 = (1 << A.shift) - 1;
    const int kgrp = (col >> 2) * 16, krow = col & 3;        /* this lane's K row: token kgrp + krow + 4 t of product t; its V: tokens 16 grp .. */
    const int qi_of = col / A.G, qh_of = col % A.G;
    struct blocks {
        int k, v;                                            /* as the table has them; -1: no token there */
    };
    /* (sixteen tokens in front of all windows are not there: their block may be another's by now, and a NaN in it times a weight of 0 is none) */
    auto read_blocks = [&](const at_spot& s) -> blocks {
        const at_request r = request(s.b);
        const int tok = (s.tile0 + s.t) * AT_TILE, low = at_from(A, r, 0) - 15;     /* (a prefix ends with a block: at a multiple of sixteen) */
        const int* pages = A.table + s.b * A.table_stride;
        auto seen = [&](int t) { return t < r.len && t >= low; };
        return {seen(tok + kgrp) ? pages[(tok + kgrp) >> A.shift] : -1, seen(tok + 16 * grp) ? pages[(tok + 16 * grp) >> A.shift] : -1};
    };
    auto place = [&](int block) { return (unsigned)block < (unsigned)A.n_blocks ? block : 0; };
    auto load_k = [&](const at_spot& s, int block, bl_v4i (&k)[4][KS]) {
        const int in = ((s.tile0 + s.t) * AT_TILE + kgrp) & bs1;
        const uint8_t* p = A.k + (((int64_t)s.h << A.shift) * D) + at_far(place(block), A.k_units) + (in + krow) * D + grp * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < KS; ++i) k[t][i] = __builtin_nontemporal_load(bl_gc<bl_v4i>(p + t * 4 * D + i * 64));
    };
    at_v4u raw[KS][2];
    auto load_q = [&](const at_spot& s) {
        const at_request R = request(s.b);
        const bool has = col < R.n * A.G;
        const uint16_t* src = A.q + (R.row0 + (has ? qi_of : 0)) * A.q_stride + (s.h * A.G + (has ? qh_of : 0)) * D;
#pragma unroll
        for (int i = 0; i < KS; ++i) raw[i][0] = *bl_gc<at_v4u>(src + i * 64 + grp * 16), raw[i][1] = *bl_gc<at_v4u>(src + i * 64 + grp * 16 + 8);
    };
    bl_v4i qh[KS], ql[KS];
    float a_row;
    auto make_pieces = [&]() {
        float most = 0.0f;
        bool odd = false;
        uint32_t w[KS][8];
#pragma unroll
        for (int i = 0; i < KS; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j] = raw[i][j >> 2][j & 3];
            most = at_largest(w[i], most, odd);
        }
        most = bl_max_pos(most, at_xor(most, 16));
        most = bl_max_pos(most, at_xor(most, 32));
        float inv, scale;
        at_row_scale<KIND>(most, inv, scale);
        const uint64_t odds = __ballot(odd);
        if (odds && ((odds >> col) & 0x0001000100010001ull)) scale = __uint_as_float(0x7fc00000u);
        a_row = scale * A.factor;
#pragma unroll
        for (int i = 0; i < KS; ++i) at_pieces<KIND>(w[i], inv, qh[i], ql[i]);
    };

    bl_v4i k[4][KS];
    load_q(cur);
    const blocks first_blocks = read_blocks(cur);
    blocks next_blocks = read_blocks(next);
    int pv = first_blocks.v;
    load_k(cur, first_blocks.k, k);
    float ks, vs;
    {
        const int64_t at = (int64_t)place(pv) * A.scale_stride + cur.h;
        ks = A.k_scale[at], vs = A.v_scale[at];
    }
    make_pieces();
    bl_v4f o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = (bl_v4f){0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    int begun = cur.t;                                       /* the item's first tile that is this wave's */
    const at_request request_kept = request(cur.b);

    for (int left = count; left > 0; --left) {
        const at_request R = request(cur.b);
        const int tok0 = (cur.tile0 + cur.t) * AT_TILE, tok = tok0 + grp * 16;    /* first of the tile's tokens, and of this lane's sixteen */
        bl_v4i v[DT];
        {
            const uint8_t* p = A.v + (((int64_t)cur.h << A.shift) * D) + at_far(place(pv), A.v_units) + ((int64_t)col << A.shift) + (tok & bs1);
            /* A tile has half of every 128-byte line of a block of 128 tokens (WIDE): the other half is to stay until the next
             * tile's turn.  Two requests of 131071 and 92681 tokens 134 -> 117 us; blocks of 64 without the hint 55 -> 60 us. */
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const bl_v4i BL_G* at = bl_gc<bl_v4i>(p + ((int64_t)(16 * i) << A.shift));
                v[i] = WIDE ? *at : __builtin_nontemporal_load(at);
            }
        }
        bl_v4f sf[4];
        if constexpr (KIND == BL_KV_INT8) {
            bl_v4i sh[4], sl[4];
            const bl_v4i z = {0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                sh[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[t][0], qh[0], z, 0, 0, 0);
                sl[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[t][0], ql[0], z, 0, 0, 0);
                if constexpr (KS == 2) {
                    sh[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[t][1], qh[1], sh[t], 0, 0, 0);
                    sl[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[t][1], ql[1], sl[t], 0, 0, 0);
                }
            }
            bl_mfma_fence();
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) sf[t][i] = (float)((sh[t][i] << 8) + sl[t][i]);   /* |.| < 2^31: exact until here */
        } else {
            at_v8i q0, q1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                q0[i] = i < 4 ? qh[0][i] : KS == 2 ? qh[KS - 1][i - 4] : 0;
                q1[i] = i < 4 ? ql[0][i] : KS == 2 ? ql[KS - 1][i - 4] : 0;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                at_v8i kk;
#pragma unroll
                for (int i = 0; i < 8; ++i) kk[i] = i < 4 ? k[t][0][i] : KS == 2 ? k[t][KS - 1][i - 4] : 0;
                sf[t] = (bl_v4f){0, 0, 0, 0};
                sf[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kk, q0, sf[t], 0, 0, 0, 0, 0, 0);
                sf[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kk, q1, sf[t], 0, 0, 0, 0, 0, 0);
            }
            bl_mfma_fence();
        }
        /* what the next tile needs, while this one computes */
        const float ks0 = ks, vs0 = vs;
        const int pv_next = next_blocks.v;
        const bool turns = !ITEM && !together && cur.t + 1 == cur.c;  /* the item ends here, and this wave goes on with the next */
        if (left > 1) {
            load_k(next, next_blocks.k, k);
            const int64_t at = (int64_t)place(pv_next) * A.scale_stride + next.h;
            ks = A.k_scale[at], vs = A.v_scale[at];
            if (turns) load_q(next);
            next_blocks = read_blocks(after);
        }
        const int qi = col < R.n * A.G ? qi_of : 0;
        const float a = a_row * ks0;
        const float vsc = fmaxf(vs0, 0x1p-100f), lv = __builtin_amdgcn_logf(vsc);
        const bool there = (unsigned)pv < (unsigned)A.n_blocks;
        const bool whole = tok0 >= at_from(A, R, R.n - 1) && tok0 + AT_TILE <= at_to(R, 0) && __all(there);
        if (!whole) {
            /* masked scores are -inf, the others have their factor already (0 * -inf is none) */
            const int see0 = at_from(A, R, qi), see1 = there && col < R.n * A.G ? at_to(R, qi) : 0;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = tok + 4 * t + i;
                    sf[t][i] = j >= see0 && j < see1 ? sf[t][i] * a : -INFINITY;
                }
        }
        float best = sf[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) best = fmaxf(best, sf[t][i]);
        best = __builtin_fmaf(best, whole ? a : 1.0f, lv);
        if (__any(best > m + AT_GROW)) {
            float top = fmaxf(m, best);
            top = fmaxf(top, at_xor(top, 16));
            top = fmaxf(top, at_xor(top, 32));
            const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
            l *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= f;
            m = top;
        }
        const float shift = at_shift(lv, m);
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sf[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sf[t][i], whole ? a : 1.0f, shift));
                sum += sf[t][i];                             /* (fp32: fp16 would lose a block whose V scale is small beside others) */
            }
        l = __builtin_fmaf(sum, __builtin_amdgcn_rcpf(vsc), l);
        const at_v4u p0 = {at_pack_half(sf[0][0], sf[0][1]), at_pack_half(sf[0][2], sf[0][3]), at_pack_half(sf[1][0], sf[1][1]), at_pack_half(sf[1][2], sf[1][3])};
        const at_v4u p1 = {at_pack_half(sf[2][0], sf[2][1]), at_pack_half(sf[2][2], sf[2][3]), at_pack_half(sf[3][0], sf[3][1]), at_pack_half(sf[3][2], sf[3][3])};
        if (!whole) {
            /* what no token has written may be anything, a NaN times 0 too */
            const int n = there ? R.len - tok : 0;
#pragma unroll
            for (int i = 0; i < DT; ++i) v[i] = at_first(v[i], n);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            at_v8h v0, v1;
            at_half16<KIND>(v[i], v0, v1);
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, __builtin_bit_cast(at_v8h, p0), o[i], 0, 0, 0);
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, __builtin_bit_cast(at_v8h, p1), o[i], 0, 0, 0);
        }
        if (turns || (!ITEM && left == 1 && !together)) {
            bl_mfma_fence();
            l += at_xor(l, 16);
            l += at_xor(l, 32);
            if (col < R.n * A.G) {
                if (turns && begun == 0) {
                    const float inv = l == 0.0f ? 0.0f : bl_div_rn(1.0f, l);
                    uint16_t* to = A.out + (R.row0 + qi_of) * A.out_stride + (cur.h * A.G + qh_of) * D + 4 * grp;
#pragma unroll
                    for (int i = 0; i < DT; ++i) {
                        const bl_v2u u = {bl_pack2_bf16(o[i][0] * inv, o[i][1] * inv), bl_pack2_bf16(o[i][2] * inv, o[i][3] * inv)};
                        *bl_g((bl_v2u*)(to + 16 * i)) = u;
                    }
                } else {
                    float* to = A.part + A.part_skip + (int64_t)(2 * stream + (begun == 0)) * at_slot<D>::floats;
#pragma unroll
                    for (int i = 0; i < DT; ++i) *bl_g((bl_v4f*)(to + col * D + 16 * i + 4 * grp)) = o[i];
                    if (grp == 0) to[AT_FEW * D + 2 * col] = m, to[AT_FEW * D + 2 * col + 1] = l;
                }
            }
            if (left > 1) {
                make_pieces();
                begun = 0, m = -INFINITY, l = 0.0f;
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = (bl_v4f){0, 0, 0, 0};
            }
        }
        if (left > 1) cur = next;
        next = after, pv = pv_next;
        if (left > 3) after = advance(after);
    }
    if (!ITEM && !together) return;
    at_meet_lds<D, WAVES>& meet = *(at_meet_lds<D, WAVES>*)lds_bytes;
    bl_mfma_fence();
    l += at_xor(l, 16);
    l += at_xor(l, 32);
    __syncthreads();                                         /* (nobody reads the requests there any more) */
    if (grp == 0) meet.m[wave][col] = m, meet.l[wave][col] = l;
#pragma unroll
    for (int i = 0; i < DT; ++i) *(bl_v4f*)&meet.o[wave][col][16 * i + 4 * grp] = o[i];
    __syncthreads();
    const at_request R = request_kept;
    constexpr int PER = D / 16;
    const int r = tid >> 4, d0 = (tid & 15) * PER;
    if (r >= R.n * A.G) return;
    float top = -INFINITY, sum = 0.0f, y[PER];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, meet.m[w][r]);
#pragma unroll
    for (int j = 0; j < PER; ++j) y[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = meet.m[w][r] == top ? 1.0f : __builtin_amdgcn_exp2f(meet.m[w][r] - top);
        sum += meet.l[w][r] * f;
#pragma unroll
        for (int j = 0; j < PER; ++j) y[j] += meet.o[w][r][d0 + j] * f;
    }
    if (SHARED && !whole_item) {
        const int64_t at = (A.group_splits + piece) * A.part_stride + at_part_at(A, at_query(A, cur.b, r / A.G), R.row0 + r / A.G, cur.h * A.G + r % A.G);
        float* to = A.many_part + at * D + d0;
#pragma unroll
        for (int j = 0; j < PER; j += 4) *bl_g((bl_v4f*)(to + j)) = (bl_v4f){y[j], y[j + 1], y[j + 2], y[j + 3]};
        if (d0 == 0) *bl_g((bl_v2f*)(A.part_ml + 2 * at)) = (bl_v2f){top, sum};
    } else if (ITEM || alone) {                              /* (SHARED: nobody else has a part of it) */
        const float inv = sum == 0.0f ? 0.0f : bl_div_rn(1.0f, sum);
        uint32_t* to = (uint32_t*)(A.out + (R.row0 + r / A.G) * A.out_stride + (cur.h * A.G + r % A.G) * D + d0);
#pragma unroll
        for (int j = 0; j < PER; j += 2) to[j / 2] = bl_pack2_bf16(y[j] * inv, y[j + 1] * inv);
    } else {
        float* to = A.part + A.part_skip + (int64_t)(2 * stream + (begun0 == 0)) * at_slot<D>::floats;
#pragma unroll
        for (int j = 0; j < PER; ++j) to[r * D + d0 + j] = y[j];
        if (d0 == 0) to[AT_FEW * D + 2 * r] = top, to[AT_FEW * D + 2 * r + 1] = sum;
    }
}

/* Adds up what several waves of at_few have of one item: of the item that the boundary between waves edge - 1 and edge cuts,
 * where no earlier boundary does.  A workgroup has AT_WAVES boundaries and the rows turn, turn + turns, ...  D / 4 threads
 * (a group) a partial result of a row.  The wave of the boundary does it, a row a group; where there are
 * more than AT_JOIN_ALONE the groups of all waves share those of a row and meet in LDS.  5 to 9 us: a kernel boundary and
 * two dependent reads of what other dies have just written.  Both launches with a bound of 8 / 32 / 128 parts, five heads of 128: one request over 4096
 * tokens 14.1 / 11.5 / 11.2 us, over 16000 17.9 / 18.0 / 21.4, over 131071 41 / 41 / 51; 16 over 8192 43.9 / 38.4 / 38.4. */
#define AT_JOIN_ALONE 32
struct at_cut {
    int row0, rows, h, first, w0, head, ga, inner, g1, parts;   /* pieces w0 .. of `head` waves, of `inner` workgroups from ga, of waves from 4 g1 */
};
struct at_sum {
    float m, l;
    bl_v4f y;
};
template <int D>
struct at_join_lds {
    float m[AT_THREADS / (D / 4)], l[AT_THREADS / (D / 4)], y[AT_THREADS / (D / 4)][D];
    at_cut cut[AT_WAVES];
};
__device__ __forceinline__ at_sum at_add(const at_sum& a, const at_sum& b) {
    at_sum r;
    r.m = fmaxf(a.m, b.m);
    const float e = a.m == r.m ? 1.0f : __builtin_amdgcn_exp2f(a.m - r.m), f = b.m == r.m ? 1.0f : __builtin_amdgcn_exp2f(b.m - r.m);
    r.l = a.l * e + b.l * f;
    r.y = a.y * e + b.y * f;
    return r;
}
/* Partial results begin, begin + step, ... of row r, features d .. d + 3, IN of them in flight. */
template <int D, int IN>
__device__ __forceinline__ at_sum at_gather(const at_args& A, const at_cut& c, int share, int r, int d, int begin, int step) {
    const float* part = A.part + A.part_skip;
    at_sum s = {-INFINITY, 0.0f, {0, 0, 0, 0}};
    for (int i = begin; i < c.parts; i += IN * step) {
        float m[IN], l[IN], best = s.m;
        bl_v4f v[IN];
#pragma unroll
        for (int u = 0; u < IN; ++u) {
            const int p = i + u * step;
            const int w = p < c.head ? c.w0 + p : p < c.head + c.inner ? (c.ga + p - c.head) * AT_WAVES : c.g1 * AT_WAVES + p - c.head - c.inner;
            const float* from = part + (int64_t)(2 * w + (w * share <= c.first)) * at_slot<D>::floats;
            m[u] = -INFINITY, l[u] = 0.0f, v[u] = (bl_v4f){0, 0, 0, 0};
            if (p < c.parts) {
                const bl_v2f ml = *bl_gc<bl_v2f>(from + AT_FEW * D + 2 * r);
                m[u] = ml[0], l[u] = ml[1];
                v[u] = *bl_gc<bl_v4f>(from + r * D + d);
            }
        }
#pragma unroll
        for (int u = 0; u < IN; ++u) best = fmaxf(best, m[u]);
        const float f = s.m == best ? 1.0f : __builtin_amdgcn_exp2f(s.m - best);
        s.l *= f, s.y *= f, s.m = best;
#pragma unroll
        for (int u = 0; u < IN; ++u) {
            const float e = m[u] == best ? 1.0f : __builtin_amdgcn_exp2f(m[u] - best);
            s.l += l[u] * e, s.y += v[u] * e;
        }
    }
    return s;
}
template <int D>
__device__ __forceinline__ void at_joined(const at_args& A, const at_cut& c, int r, int d, const at_sum& s) {
    const float inv = s.l == 0.0f ? 0.0f : bl_div_rn(1.0f, s.l);
    const bl_v2u u = {bl_pack2_bf16(s.y[0] * inv, s.y[1] * inv), bl_pack2_bf16(s.y[2] * inv, s.y[3] * inv)};
    *bl_g((bl_v2u*)(A.out + (c.row0 + r / A.G) * A.out_stride + (c.h * A.G + r % A.G) * D + d)) = u;
}
template <int D, int IN>
__device__ __forceinline__ void at_few_join(const at_args& A, int group, int turn, int turns, at_join_lds<D>& lds) {
    constexpr int TPP = D / 4, GROUPS = AT_THREADS / TPP, PER_WAVE = GROUPS / AT_WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = at_uniform(tid >> 6), d = tid % TPP * 4;
    const int4* heads = (const int4*)A.part;
    /* 64 requests at a look: the first whose tiles end behind tile `at` of a head's line is this boundary's */
    int4 here = {0, 0, 0, 0};
    int total, b0 = 0;
    const bool small = A.B <= 64;
    if (small) {
        here = heads[lane < A.B ? lane : A.B - 1];
        total = __builtin_amdgcn_readlane(here.x, 63);
    } else {
        total = heads[A.B - 1].x;
    }
    const int all = total * A.n_kv, share = at_share(all), edge = group * AT_WAVES + wave + 1;
    if ((int64_t)(group * AT_WAVES + 1) * share >= all) return;
    at_cut c = {};
    if ((int64_t)edge * share < all) {
        const int pos = edge * share, at = pos / A.n_kv;
        if (!small) {
            const int i = lane * 64 + 63;
            b0 = __builtin_ctzll(__ballot(heads[i < A.B ? i : A.B - 1].x > at)) * 64;
            here = heads[b0 + lane < A.B ? b0 + lane : A.B - 1];
        }
        const int i = __builtin_ctzll(__ballot(here.x > at));
        const int before = i ? __builtin_amdgcn_readlane(here.x, i - 1) : b0 ? at_uniform(heads[b0 - 1].x) : 0;
        const int n = __builtin_amdgcn_readlane(here.x, i) - before;
        c.h = (pos - before * A.n_kv) / n, c.first = before * A.n_kv + c.h * n;
        const int last = c.first + n - 1, w1 = last / share;
        c.w0 = c.first / share;
        const int g0 = c.w0 / AT_WAVES;
        c.g1 = w1 / AT_WAVES;
        const bool in0 = at_together(g0, share, c.first, last), in1 = at_together(c.g1, share, c.first, last);
        c.head = in0 ? 0 : (w1 < g0 * AT_WAVES + AT_WAVES - 1 ? w1 : g0 * AT_WAVES + AT_WAVES - 1) - c.w0 + 1;
        c.ga = in0 ? g0 : g0 + 1;
        c.inner = (in1 ? c.g1 + 1 : c.g1) - c.ga;
        c.inner = c.inner < 0 ? 0 : c.inner;
        c.parts = c.head + c.inner + (in1 || c.g1 == g0 ? 0 : w1 - c.g1 * AT_WAVES + 1);
        if (c.w0 != edge - 1) c.parts = 0;                               /* not this boundary's */
        c.row0 = __builtin_amdgcn_readlane(here.y, i), c.rows = __builtin_amdgcn_readlane(here.z, i) * A.G;
    }
    const bool together = c.parts > AT_JOIN_ALONE;
    if (!together && c.parts > 1)
        for (int r = turn * PER_WAVE + lane / TPP; r < c.rows; r += turns * PER_WAVE) at_joined<D>(A, c, r, d, at_gather<D, IN>(A, c, share, r, d, 0, 1));
    if (lane == 0) {
        if (!together) c.rows = 0;
        lds.cut[wave] = c;
    }
    __syncthreads();
    for (int i = 0; i < AT_WAVES; ++i) {
        const at_cut x = lds.cut[i];
        for (int r = turn; r < x.rows; r += turns) {
            const int g = tid / TPP;
            at_sum s = at_gather<D, IN>(A, x, share, r, d, g, GROUPS);
            if (d == 0) lds.m[g] = s.m, lds.l[g] = s.l;
            *(bl_v4f*)&lds.y[g][d] = s.y;
            __syncthreads();
            if (g == 0) {
                for (int j = 1; j < GROUPS; ++j) s = at_add(s, {lds.m[j], lds.l[j], *(const bl_v4f*)&lds.y[j][d]});
                at_joined<D>(A, x, r, d, s);
            }
            __syncthreads();
        }
    }
}

/* ---- many rows: the matrix cores work -------------------------------------------------------------------------------- */

__device__ __forceinline__ int at_many_tiles(const at_args& A, int b) {
    const at_request r = at_read(A, b);
    const int64_t rows = (int64_t)r.n * A.G;
    return rows > A.few_rows ? (int)((rows + AT_MANY - 1) / AT_MANY) : 0;
}

/* A workgroup: 128 rows of one request and kv head, 32 a wave, over a range of its tiles (all that its rows see, or one of
 * `splits` equal pieces).  V lies in LDS as fp16, converted once by the thread that
 * loads it, K as its codes, which the matrix cores multiply with the two pieces of q, or (int8, heads of 64) as fp16 too: the pieces'
 * products cost two vector instructions a score more, their conversion is one instruction for half a byte, and a third wave fits (8000
 * tokens, 32 + 8 heads: 417 -> 369 us; heads of 128: 388 -> 401, LDS reads).  16-byte units are XOR-ed with the row, so that sixteen
 * lanes of a read fall on all 64 banks; two buffers, one barrier a tile.
 * Bound by vector instructions (376 a wave and tile beside 1024 matrix clocks; vector units busy 52 % of the time, matrix cores
 * 32 %) where the workgroups are many: 8000 tokens of 20 + 5 heads of 128 832 TFLOP/s, e4m3 911 (a library bf16 product of 8192^3: 1224).  A prompt of
 * 4096: 121 us = 711, where the last rows' 64 tiles one after the other are all of it; cutting them in two took 145 us (the halves' 42 MB).  Products of 32 tokens x
 * 32 rows (S^T) and 32 features x 32 rows (O^T): a lane has one row. */
template <int KIND, int D>
struct at_many_k {                  /* bytes of a K value in LDS */
    static constexpr int bytes = KIND == BL_KV_INT8 && D == 64 ? 2 : 1;
};
template <int KIND, int D>
struct at_many_lds {
    union {
        uint8_t v[2][D * AT_TILE * 2];
        int upto[BL_KV_MAX_REQUESTS];                       /* at first */
    };
    uint8_t k[2][AT_TILE * D * at_many_k<KIND, D>::bytes];
    int scan[AT_WAVES];
};
template <int KIND, int D>
struct at_prefix_lds : at_many_lds<KIND, D> {
    int2 query[AT_MANY];                                    /* row and position of the tile's queries, */
    int slot[AT_MANY];                                      /* and at_query */
    int2 ends[AT_WAVES];
    int found[5];                                           /* the group of the tile, tiles in front of it and of it, its tokens and rows */
};
/* What a workgroup of at_many has: rows of a request over all that they see; over what stands behind their group's prefix (AT_OWN); or rows of all
 * requests of a group over its prefix (AT_PREFIX), which are gathered: their places in the batch are found by each workgroup, by sums over the requests.
 * A prefix's rows fill tiles together (128 of them for one read of K and V), in equal pieces over its tokens, so that every row of a group has as many partial results and
 * the join needs no list.  Not bound by memory, nor by any one of a tile's parts: 16 requests of 32 + 8 heads behind 65536 tokens, e4m3, 134 MB of codes,
 * 50 us, without loads 47, without products 40: a wave's tiles one after the other, on two waves a SIMD (at_few reads them for each request: 337).  Two tiles of K in flight, pairs
 * of waves on one tile's rows: 49 and 47. */
enum { AT_ALL, AT_OWN, AT_PREFIX };
template <int KIND, int D, int MODE = AT_ALL>
__device__ __forceinline__ void at_many(const at_args& A, int place, std::conditional_t<MODE == AT_PREFIX, at_prefix_lds<KIND, D>, at_many_lds<KIND, D>>& lds) {
    const int splits = MODE == AT_PREFIX ? A.group_splits : MODE == AT_OWN ? A.many_splits : A.splits;
    constexpr bool HALF = at_many_k<KIND, D>::bytes == 2;
    constexpr int KROW = D * at_many_k<KIND, D>::bytes;        /* bytes of a K row in LDS, 16-byte units XOR-ed by k_mix(row) */
    constexpr int KS = D / 32, DT = D / 32;
    auto k_mix = [](int row) { return KROW == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
    auto& s_k = lds.k;
    auto& s_v = lds.v;
    const int tid = threadIdx.x, lane = tid & 63, wave = at_uniform(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    /* whose tile: place = (row tile * n_kv + head) * splits + piece, a request's heavy tiles first */
    int piece, h, want, b, before, c, rt;
    auto take = [&](int all) {
        /* Heads of 128: of the 512 workgroups that the chip holds the second 256 go the other way round, so that a unit has a heavy
         * one and a light one: two prompts of 1600 tokens 72 -> 57 us, one of 6000 244 -> 236 (heads of 64, three to a unit: 52 -> 58). */
        const int n = all * A.n_kv * splits, both = n < 512 ? n : 512;
        if (D == 128 && place >= 256 && place < both) place = 255 + both - place;
        piece = place % splits, h = place / splits % A.n_kv, want = place / splits / A.n_kv;
        return place < n;
    };
    at_request R = {};
    int group_rows = 0;
    if constexpr (MODE == AT_PREFIX) {
        int* s_upto = lds.upto;
        /* Which group has this tile, and the batch rows of the tile's queries: sums over the groups, then over the requests.  A thread has one of each where there
         * are no more than threads, so that all of it hangs on one round of loads. */
        auto queries = [&](int q0, int q1, int begin, int end, int request, int row0, int len) {
            for (int j = begin > q0 ? begin : q0; j < (end < q1 ? end : q1); ++j)
                lds.query[j - q0] = make_int2(row0 + j - begin, len - (end - begin) + j - begin), lds.slot[j - q0] = at_query(A, request, j - begin);
        };
        auto range = [&](int& q0, int& q1) {
            rt = c - 1 - (want - before);
            q0 = rt * AT_MANY / A.G, q1 = (rt * AT_MANY + AT_MANY - 1) / A.G + 1;
        };
        if (A.B <= AT_THREADS && A.n_groups <= AT_THREADS) {
            int group = -1, tokens = 0;
            at_request r = {};
            if (tid < A.B) group = A.group[tid], r = at_read(A, tid);
            if (tid < A.n_groups) tokens = at_shared_tokens(A, tid);
            if ((unsigned)group >= (unsigned)A.n_groups || !at_grouped(A, r.n)) r.n = 0;
            s_upto[tid] = 0;
            __syncthreads();
            if (r.n) atomicAdd(&s_upto[group], r.n);
            __syncthreads();
            const int rows = s_upto[tid] * A.G, tiles = tokens ? (rows + AT_MANY - 1) / AT_MANY : 0;
            auto sums = [&](int v, int* total) {             /* over the threads up to this one */
                const int x = at_scan(v);
                if (lane == 63) lds.scan[wave] = x;
                __syncthreads();
                int add = 0, all = 0;
#pragma unroll
                for (int w = 0; w < AT_WAVES; ++w) add += w < wave ? lds.scan[w] : 0, all += lds.scan[w];
                *total = all;
                return x + add;
            };
            int all;
            const int upto = sums(tiles, &all);
            if (!take(at_uniform(all))) return;
            if (tiles && upto > want && upto - tiles <= want) lds.found[0] = tid, lds.found[1] = upto - tiles, lds.found[2] = tiles, lds.found[3] = tokens, lds.found[4] = rows;
            __syncthreads();
            b = at_uniform(lds.found[0]), before = at_uniform(lds.found[1]), c = at_uniform(lds.found[2]);
            R.len = at_uniform(lds.found[3]), group_rows = at_uniform(lds.found[4]);
            int q0, q1;
            range(q0, q1);
            const int n = group == b ? r.n : 0, end = sums(n, &all);
            if (n) queries(q0, q1, end - n, end, tid, r.row0, r.len);
            __syncthreads();
        } else {
            auto news = [&](int i) {
                const int n = at_read(A, i).n;
                return at_grouped(A, n) ? n : 0;
            };
            for (int g = tid; g < A.n_groups; g += AT_THREADS) s_upto[g] = 0;
            __syncthreads();
            for (int i = tid; i < A.B; i += AT_THREADS) {
                const int g = A.group[i], n = news(i);
                if ((unsigned)g < (unsigned)A.n_groups && n) atomicAdd(&s_upto[g], n);
            }
            __syncthreads();
            at_sums(A.n_groups, [&](int g) { return at_shared_tokens(A, g) ? (int)(((int64_t)s_upto[g] * A.G + AT_MANY - 1) / AT_MANY) : 0; }, s_upto, lds.scan);
            if (!take(at_uniform(s_upto[A.n_groups - 1]))) return;
            int lo = -1, hi = A.n_groups - 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_upto[mid] > want) hi = mid;
                else lo = mid;
            }
            b = at_uniform(hi);
            before = b ? at_uniform(s_upto[b - 1]) : 0;
            c = at_uniform(s_upto[b]) - before;
            R.len = at_shared_tokens(A, b);
            __syncthreads();
            at_sums(A.B, [&](int i) { return A.group[i] == b ? news(i) : 0; }, s_upto, lds.scan);
            group_rows = at_uniform(s_upto[A.B - 1]) * A.G;
            int q0, q1;
            range(q0, q1);
            for (int i = tid; i < A.B; i += AT_THREADS) {
                const int end = s_upto[i], begin = i ? s_upto[i - 1] : 0;
                if (end <= q0 || begin >= q1 || end == begin) continue;
                const at_request r = at_read(A, i);
                queries(q0, q1, begin, end, i, r.row0, r.len);
            }
            __syncthreads();
        }
    } else if (A.B <= 64) {
        const int upto = at_scan(lane < A.B ? at_many_tiles(A, lane) : 0);
        if (!take(__builtin_amdgcn_readlane(upto, 63))) return;
        b = __builtin_ctzll(__ballot(upto > want));
        before = b ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        c = __builtin_amdgcn_readlane(upto, b) - before;
    } else {
        int* s_upto = lds.upto;
        at_sums(A.B, [&](int i) { return at_many_tiles(A, i); }, s_upto, lds.scan);
        if (!take(at_uniform(s_upto[A.B - 1]))) return;
        int lo = -1, hi = A.B - 1;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_upto[mid] > want) hi = mid;
            else lo = mid;
        }
        b = at_uniform(hi);
        before = b ? at_uniform(s_upto[b - 1]) : 0;
        c = at_uniform(s_upto[b]) - before;
        __syncthreads();
    }
    const int bs1 = (1 << A.shift) - 1;
    int rows;
    if constexpr (MODE == AT_PREFIX) {
        rows = group_rows;
    } else {
        rt = c - 1 - (want - before);                        /* the last rows see most: first */
        R = at_read_own<MODE == AT_OWN>(A, b);
        rows = R.n * A.G;
        if (MODE == AT_OWN && !at_grouped(A, R.n)) R.skip = 0;
    }
    const int rbase = rt * AT_MANY, rend = rbase + AT_MANY < rows ? rbase + AT_MANY : rows;
    /* tokens that some row of the workgroup sees (asked for here, in front of what differs by lane: behind it the compiler keeps the bounds in vector
     * registers, and a prompt of 4096 tokens takes 128 us for 123) */
    int tok0 = 0, tok1 = 0;
    if constexpr (MODE != AT_PREFIX) tok0 = at_from(A, R, rbase / A.G), tok1 = at_to(R, (rend - 1) / A.G);
    /* this lane's row: its place in the batch, its head, and the tokens that it sees */
    const int row = rbase + wave * 32 + col;
    const bool live = row < rows;
    const int qi = live ? row / A.G : 0, qh_i = h * A.G + (live ? row % A.G : 0);
    int at_row, see0, see1, slot = 0;
    if constexpr (MODE == AT_PREFIX) {
        const int2 q = lds.query[live ? qi - rbase / A.G : 0];
        slot = lds.slot[live ? qi - rbase / A.G : 0];
        const int from = A.window ? q.y - A.window + 1 : 0;
        at_row = q.x, see0 = from > 0 ? from : 0, see1 = !live || q.y < 0 ? 0 : q.y + 1 < R.len ? q.y + 1 : R.len;
    } else {
        at_row = R.row0 + qi, see0 = at_from(A, R, qi), see1 = live ? at_to(R, qi) : 0;
    }
    /* tokens that some row of this wave sees, and that all do */
    const int wfirst = rbase + wave * 32, wlast = wfirst + 31 < rows ? wfirst + 31 : rows - 1;
    const bool has_rows = wfirst < rows;
    int any_from, any_to, all_from, all_to;
    if constexpr (MODE == AT_PREFIX) {
        any_from = all_from = see0, any_to = all_to = see1;
        if (!live) any_from = all_to = 0x7fffffff, all_from = any_to = 0;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
            any_from = min(any_from, __shfl_xor(any_from, x)), any_to = max(any_to, __shfl_xor(any_to, x));
            all_from = max(all_from, __shfl_xor(all_from, x)), all_to = min(all_to, __shfl_xor(all_to, x));
        }
        any_from = at_uniform(any_from), any_to = at_uniform(any_to), all_from = at_uniform(all_from), all_to = at_uniform(all_to);
        if (lane == 0) lds.ends[wave] = make_int2(any_from, any_to);
        __syncthreads();
        tok0 = 0x7fffffff, tok1 = 0;
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) tok0 = min(tok0, lds.ends[w].x), tok1 = max(tok1, lds.ends[w].y);
        tok0 = at_uniform(tok0), tok1 = at_uniform(tok1);
    } else {
        any_from = has_rows ? at_from(A, R, wfirst / A.G) : 0, any_to = has_rows ? at_to(R, wlast / A.G) : 0;
        all_from = has_rows ? at_from(A, R, wlast / A.G) : 0, all_to = has_rows ? at_to(R, wfirst / A.G) : 0;
    }
    int tile = tok0 / AT_TILE, tend = (tok1 + AT_TILE - 1) / AT_TILE;
    if (tend < tile) tend = tile;
    if constexpr (MODE == AT_PREFIX) {
        /* equal pieces of the whole prefix, so that every row of the group has the same */
        const int all = (R.len + AT_TILE - 1) / AT_TILE, n = at_piece(all, splits);
        if (piece * n >= all) return;
        tile = max(tile, piece * n), tend = min(tend, piece * n + n);
    } else {
        const int n = (tend - tile + splits - 1) / splits;
        tile += piece * n;
        tend = tile + n < tend ? tile + n : tend;
    }
    const int* pages = MODE == AT_PREFIX ? A.shared_table + b * A.shared_stride : A.table + b * A.table_stride;
    /* this lane's part of q: as fp16 (HALF: values d = 16 s + 8 half .. + 7, times a power of two, exact down to 2^-27 of the
     * row's largest), or as two 8-bit pieces (values d = 32 s + 16 half .. + 15) */
    at_v8h qf[2 * KS];
    bl_v4i qh[KS], ql[KS];
    float a_row;
    {
        uint32_t w[KS][8];
        const uint16_t* src = A.q + at_row * A.q_stride + qh_i * D;
        float most = 0.0f;
        bool odd = false;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const at_v4u u0 = *bl_gc<at_v4u>(src + s * 32 + half * (HALF ? 8 : 16)), u1 = *bl_gc<at_v4u>(src + s * 32 + (HALF ? 16 + half * 8 : half * 16 + 8));
#pragma unroll
            for (int j = 0; j < 4; ++j) w[s][j] = u0[j], w[s][4 + j] = u1[j];
            most = at_largest(w[s], most, odd);
        }
        most = bl_max_pos(most, at_xor(most, 32));
        float inv, scale;
        if (HALF) at_power_scale(most, 137, inv, scale);
        else at_row_scale<KIND>(most, inv, scale);
        const uint64_t odds = __ballot(odd);
        if (odds && ((odds >> col) & 0x0000000100000001ull)) scale = __uint_as_float(0x7fc00000u);
        a_row = scale * A.factor;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if constexpr (HALF) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    at_v4u t;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t v = w[s][4 * x + j];
                        t[j] = at_pack_half(bl_bf16_to_f32(v & 0xffffu) * inv, __uint_as_float(v & 0xffff0000u) * inv);
                    }
                    qf[2 * s + x] = __builtin_bit_cast(at_v8h, t);
                }
            } else {
                at_pieces<KIND>(w[s], inv, qh[s], ql[s]);
            }
        }
    }
    at_v16f o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    const int64_t head = ((int64_t)h << A.shift) * D;
    /* Loading: a wave's sixteen tokens, D/64 16-byte units of K and of V a lane.  They lie in one block, so that the block's place is
     * a scalar and the lanes' offsets never change.  A tile's blocks are read two tiles ahead (lane g: the block of its
     * tokens 16g..), its codes and scales one tile ahead: no load waits for another's address. */
    constexpr int U = D / 64;
    const int kt = lane >> 2, kc = (lane & 3) * U;           /* K: four lanes a row */
    const int k_off = kt * D + kc * 16, v_off = lane << A.shift;          /* V: features lane and lane + 64 */
    auto fetch_blocks = [&](int t) -> int {
        const int token = t * AT_TILE + 16 * (lane & 3);
        return t < tend && token < R.len && token + 16 > tok0 ? pages[token >> A.shift] : -1;       /* (in front of all windows: as in at_few) */
    };
    auto there = [&](int block) { return (unsigned)block < (unsigned)A.n_blocks; };
    bl_v4i lk[U], lv_[U];
    float ks_next = 0.0f, vs_next = 0.0f;
    auto load = [&](int t, int blocks) {
        const int mine = __builtin_amdgcn_readlane(blocks, wave), in = (t * AT_TILE + 16 * wave) & bs1;
        const uint8_t* kp = A.k + head + at_far(there(mine) ? mine : 0, A.k_units) + in * D;
        const uint8_t* vp = A.v + head + at_far(there(mine) ? mine : 0, A.v_units) + in;
#pragma unroll
        for (int u = 0; u < U; ++u) lk[u] = *bl_gc<bl_v4i>(kp + k_off + u * 16);
#pragma unroll
        for (int u = 0; u < U; ++u) lv_[u] = *bl_gc<bl_v4i>(vp + v_off + (u * 64 << A.shift));
        const int64_t sc = (int64_t)(there(blocks) ? blocks : 0) * A.scale_stride + h;
        ks_next = A.k_scale[sc], vs_next = A.v_scale[sc];
    };
    const int k_row = 16 * wave + kt, k_swz = k_mix(k_row);
    /* What no token has written may be anything, and a NaN times 0 is none: zeros behind the last token of tile t. */
    auto mend = [&](int t, int blocks) {
        const int n = there(__builtin_amdgcn_readlane(blocks, wave)) ? R.len - t * AT_TILE - 16 * wave : 0;
        if (n < 16)
#pragma unroll
            for (int u = 0; u < U; ++u) lv_[u] = at_first(lv_[u], n);
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at_v8h a, c;
            if constexpr (HALF) {
                at_half16<KIND>(lk[u], a, c);
                *(at_v8h*)&s_k[buf][k_row * KROW + (((2 * (kc + u)) ^ k_swz) * 16)] = a;
                *(at_v8h*)&s_k[buf][k_row * KROW + (((2 * (kc + u) + 1) ^ k_swz) * 16)] = c;
            } else {
                *(bl_v4i*)&s_k[buf][k_row * KROW + (((kc + u) ^ k_swz) * 16)] = lk[u];
            }
            at_half16<KIND>(lv_[u], a, c);
            const int d = lane + 64 * u;
            *(at_v8h*)&s_v[buf][d * 128 + (((2 * wave) ^ ((d >> 1) & 7)) * 16)] = a;
            *(at_v8h*)&s_v[buf][d * 128 + (((2 * wave + 1) ^ ((d >> 1) & 7)) * 16)] = c;
        }
    };
    /* of the tile computed and of the next two */
    int blk0 = fetch_blocks(tile), blk1 = fetch_blocks(tile + 1), blk2 = fetch_blocks(tile + 2);
    float ks_v = 0.0f, vs_v = 0.0f, ks_1 = 0.0f, vs_1 = 0.0f;
    if (tile < tend) {
        load(tile, blk0);
        ks_v = ks_next, vs_v = vs_next;
        mend(tile, blk0);
        store(0);
        load(tile + 1, blk1);
        ks_1 = ks_next, vs_1 = vs_next;
    }
    __syncthreads();
    /* row r = 8a + 4f + b of the first product's tile tt is token 32 tt + 16 (a/2) + 8 f + 4 (a%2) + b */
    const int kr = (col >> 4) * 16 + ((col >> 2) & 1) * 8 + ((col >> 3) & 1) * 4 + (col & 3);
    const int kr_swz = k_mix(kr);
    /* One step: the next tile goes to LDS and the one's behind it is asked for while the first product runs, and each group's
     * weights are made while the one's before it are multiplied. */
    for (int buf = 0; tile < tend; ++tile, buf ^= 1) {
        const int tok = tile * AT_TILE;
        const int blk3 = fetch_blocks(tile + 3);
        mend(tile + 1, blk1);
        if (tok < any_to && tok + AT_TILE > any_from) {
            float sf[2][16];
            auto v_part = [&](int g, int i) { return *(const at_v8h*)&s_v[buf][(32 * i + col) * 128 + (((2 * g + half) ^ ((col >> 1) & 7)) * 16)]; };
            auto k_part = [&](int tt, int i) { return *(const bl_v4i*)&s_k[buf][(tt * 32 + kr) * KROW + (((2 * i + half) ^ kr_swz) * 16)]; };
            at_v8h vv[2][DT];
            constexpr int UNITS = KROW / 32;                 /* a lane's 16-byte units of a K row */
            bl_v4i kk[2][UNITS];
#pragma unroll
            for (int i = 0; i < UNITS; ++i) kk[0][i] = k_part(0, i), kk[1][i] = k_part(1, i);
            if constexpr (KIND == BL_KV_INT8 && !HALF) {
                /* the second half's products run over the first half's conversion */
                bl_v16i sh[2], sl[2];
#pragma unroll
                for (int j = 0; j < 16; ++j) sh[0][j] = sl[0][j] = sh[1][j] = sl[1][j] = 0;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    sh[0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[0][s], qh[s], sh[0], 0, 0, 0);
                    sl[0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[0][s], ql[s], sl[0], 0, 0, 0);
                }
                store(buf ^ 1);
#pragma unroll
                for (int s = 0; s < 2 * KS; ++s) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, D / 16, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                sh[1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[1][0], qh[0], sh[1], 0, 0, 0);
                sl[1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[1][0], ql[0], sl[1], 0, 0, 0);
                load(tile + 2, blk2);
                __builtin_amdgcn_sched_barrier(0);          /* (two products between the first half's last and its first reader) */
#pragma unroll
                for (int s = 1; s < KS; ++s) {
                    sh[1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[1][s], qh[s], sh[1], 0, 0, 0);
                    sl[1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kk[1][s], ql[s], sl[1], 0, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) sf[0][j] = (float)((sh[0][j] << 8) + sl[0][j]);
#pragma unroll
                for (int s = 2; s < 2 * KS; ++s) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 32 / (2 * KS - 2) + 1, 0);
                }
                bl_mfma_fence();
#pragma unroll
                for (int i = 0; i < DT; ++i) vv[0][i] = v_part(0, i);
#pragma unroll
                for (int j = 0; j < 16; ++j) sf[1][j] = (float)((sh[1][j] << 8) + sl[1][j]);
            } else {
                at_v16f s16[2];
#pragma unroll
                for (int j = 0; j < 16; ++j) s16[0][j] = s16[1][j] = 0.0f;
                constexpr int STEPS = HALF ? 2 * KS : KS / 2, EACH = HALF ? 2 : 4;      /* k steps, products of one */
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    if constexpr (HALF) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) s16[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(at_v8h, kk[u][s]), qf[s], s16[u], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            at_v8i ka, qa;
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                ka[j] = kk[u & 1][2 * s + j / 4][j % 4], qa[j] = u < 2 ? qh[2 * s + j / 4][j % 4] : ql[2 * s + j / 4][j % 4];
                            s16[u & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qa, s16[u & 1], 0, 0, 0, 0, 0, 0);
                        }
                    }
                }
                store(buf ^ 1);
                load(tile + 2, blk2);
#pragma unroll
                for (int i = 0; i < DT; ++i) vv[0][i] = v_part(0, i);
#pragma unroll
                for (int s = 0; s < STEPS * EACH; ++s) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, HALF ? 6 : D / 16, 0);
                }
                bl_mfma_fence();
#pragma unroll
                for (int j = 0; j < 16; ++j) sf[0][j] = s16[0][j], sf[1][j] = s16[1][j];
            }
            const float vs_c = fmaxf(vs_v, 0x1p-100f), lv_v = __builtin_amdgcn_logf(vs_c), rv_v = __builtin_amdgcn_rcpf(vs_c);
            const unsigned groups = (unsigned)__ballot(there(blk0)) & 15u;
            const bool whole = groups == 15u && tok >= all_from && tok + AT_TILE <= all_to;
            float a[4], lv[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) a[g] = a_row * bl_lane_f(ks_v, g), lv[g] = bl_lane_f(lv_v, g);
            if (!whole) {
                /* masked scores are -inf, the others have their factor already (0 * -inf is none) */
#pragma unroll
                for (int g = 0; g < 4; ++g) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float& x = sf[g >> 1][(g & 1) * 8 + j];
                        const int t = tok + 16 * g + 8 * half + j;
                        x = (groups >> g & 1) && t >= see0 && t < see1 ? x * a[g] : -INFINITY;
                    }
                    a[g] = 1.0f;
                }
            }
            float best = -INFINITY;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float top = sf[g >> 1][(g & 1) * 8];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, sf[g >> 1][(g & 1) * 8 + j]);
                best = fmaxf(best, __builtin_fmaf(top, a[g], lv[g]));
            }
            if (__any(best > m + AT_GROW)) {
                float top = fmaxf(m, best);
                top = fmaxf(top, at_xor(top, 32));
                const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
                l *= f;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= f;
                m = top;
            }
            auto weights = [&](int g) {
                const float shift = at_shift(lv[g], m);
                float w[8], sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sf[g >> 1][(g & 1) * 8 + j], a[g], shift));
                    sum += w[j];                             /* (fp32: fp16 would lose a block whose V scale is small beside others) */
                }
                l = __builtin_fmaf(sum, bl_lane_f(rv_v, g), l);
                return __builtin_bit_cast(at_v8h, (at_v4u){at_pack_half(w[0], w[1]), at_pack_half(w[2], w[3]), at_pack_half(w[4], w[5]), at_pack_half(w[6], w[7])});
            };
            at_v8h p = weights(0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                at_v8h next = p;
                if (g < 3) {
#pragma unroll
                    for (int i = 0; i < DT; ++i) vv[(g + 1) & 1][i] = v_part(g + 1, i);
                }
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv[g & 1][i], p, o[i], 0, 0, 0);
                if (g < 3) {
                    next = weights(g + 1);
                    __builtin_amdgcn_sched_group_barrier(0x100, DT, 0);
#pragma unroll
                    for (int i = 0; i < DT; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 32 / DT + 1, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                p = next;
            }
        } else {
            store(buf ^ 1);
            load(tile + 2, blk2);
        }
        blk0 = blk1, blk1 = blk2, blk2 = blk3;
        ks_v = ks_1, vs_v = vs_1, ks_1 = ks_next, vs_1 = vs_next;
        __syncthreads();
    }
    bl_mfma_fence();
    l += at_xor(l, 32);
    if (!live) return;
    const bool whole_rows = MODE == AT_ALL ? A.splits == 1 : MODE == AT_OWN && R.skip == 0 && splits == 1;
    if (MODE == AT_OWN && h == 0 && piece == 0 && half == 0 && row % A.G == 0)
        A.pieces[at_row] = make_int2(whole_rows ? 0 : at_pieces(at_piece_count((R.skip + AT_TILE - 1) / AT_TILE, A.group_splits), splits, true), R.skip ? at_query(A, b, qi) : 0);
    if (whole_rows) {
        const float inv = l == 0.0f ? 0.0f : bl_div_rn(1.0f, l);
        uint16_t* to = A.out + at_row * A.out_stride + qh_i * D;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const bl_v2u u = {bl_pack2_bf16(o[i][j] * inv, o[i][j + 1] * inv), bl_pack2_bf16(o[i][j + 2] * inv, o[i][j + 3] * inv)};
                *bl_g((bl_v2u*)(to + 32 * i + 2 * j + 4 * half)) = u;
            }
    } else {
        const int64_t at = MODE == AT_PREFIX ? piece * A.part_stride + at_part_at(A, slot, at_row, qh_i)
                                             : (MODE == AT_OWN ? A.own_at : 0) + ((int64_t)piece * A.T + at_row) * A.n_q + qh_i;
        float* to = A.many_part + at * D;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) *bl_g((bl_v4f*)(to + 32 * i + 2 * j + 4 * half)) = (bl_v4f){o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]};
        if (half == 0) {
            float* ml = (MODE == AT_ALL ? A.many_part + (int64_t)A.splits * A.T * A.n_q * D : A.part_ml) + 2 * at;
            ml[0] = m, ml[1] = l;
        }
    }
}

/* Adds up the pieces of a split: D / 4 threads a (row of the batch, head), four pieces in flight. */
template <int D>
__device__ __forceinline__ void at_many_join(const at_args& A, int group) {
    constexpr int TPR = D / 4, IN = 4;
    const int64_t at = (int64_t)group * (AT_THREADS / TPR) + threadIdx.x / TPR, all = (int64_t)A.T * A.n_q;
    if (at >= all) return;
    const int row = (int)(at / A.n_q), d0 = (threadIdx.x % TPR) * 4;
    const float* ml = A.many_part + A.splits * all * D;
    auto piece = [&](int i) -> at_sum {
        at_sum x = {-INFINITY, 0.0f, {0, 0, 0, 0}};
        if (i < A.splits) {
            const int64_t from = i * all + at;
            const bl_v2f t = *bl_gc<bl_v2f>(ml + 2 * from);
            x.m = t[0], x.l = t[1], x.y = *bl_gc<bl_v4f>(A.many_part + from * D + d0);
        }
        return x;
    };
    at_sum x[IN];
#pragma unroll
    for (int u = 0; u < IN; ++u) x[u] = piece(u);
    int lo = 0, hi = A.B;                                     /* whose row it is, while those come: q_start[lo] <= row < q_start[hi] */
    if (row < A.q_start[0] || row >= A.q_start[A.B]) return;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (A.q_start[mid] <= row) lo = mid;
        else hi = mid;
    }
    const at_request R = at_read(A, lo);
    if ((int64_t)R.n * A.G <= A.few_rows) return;
    at_sum s = x[0];
#pragma unroll
    for (int u = 1; u < IN; ++u) s = at_add(s, x[u]);
    for (int i = IN; i < A.splits; i += IN) {
#pragma unroll
        for (int u = 0; u < IN; ++u) x[u] = piece(i + u);
#pragma unroll
        for (int u = 0; u < IN; ++u) s = at_add(s, x[u]);
    }
    const float inv = s.l == 0.0f ? 0.0f : bl_div_rn(1.0f, s.l);
    const bl_v2u u = {bl_pack2_bf16(s.y[0] * inv, s.y[1] * inv), bl_pack2_bf16(s.y[2] * inv, s.y[3] * inv)};
    *bl_g((bl_v2u*)(A.out + row * A.out_stride + (at % A.n_q) * D + d0)) = u;
}

/* The same for rows of requests that share prefixes: the pieces of the prefix and those of the rest, as many as the row's entry says.  LANES groups of
 * D / 4 threads share a row's pieces and meet in LDS.  Bound by the chain entry -> references -> sums: 64 rows of 20 heads, 16 + 4 pieces, 5.0 us; 16 of 32, 64 + 2, 6.7. */
template <int D, int LANES>
__global__ __launch_bounds__(AT_THREADS) void bl_attn_shared_join(at_args A) {
    constexpr int TPR = D / 4, IN = 4, GROUPS = AT_THREADS / TPR, ROWS = GROUPS / LANES;
    __shared__ float s_m[GROUPS], s_l[GROUPS];
    __shared__ __attribute__((aligned(16))) float s_y[GROUPS][D];
    const int group = threadIdx.x / TPR, part = group / ROWS;               /* (a wave's groups have other rows: their loads are of neighbours) */
    const uint32_t at = blockIdx.x * ROWS + group % ROWS, all = (uint32_t)A.T * A.n_q;                  /* (below 2^28) */
    const int row = (int)(at / (uint32_t)A.n_q), head = (int)(at % (uint32_t)A.n_q), d0 = (threadIdx.x % TPR) * 4;
    int2 entry = {0, 0};
    if (at < all) entry = A.pieces[row];
    if (row < A.q_start[0] || row >= A.q_start[A.B]) entry = {0, 0};
    if (LANES == 1 && entry.x == 0) return;
    /* (first rows that do not ascend leave entries unwritten: no content of them leads outside) */
    const bool none = entry.x == AT_NO_NUMBERS, many = entry.x >> 16 & 1;
    const int prefix = none ? 0 : min(entry.x & 255, A.G < A.apart ? A.group_splits : 0), own = none ? 0 : min(entry.x >> 8 & 255, many ? A.many_splits : A.few_splits), count = prefix + own;
    const int slot = (unsigned)entry.y < (unsigned)(A.B * A.apart) && (entry.y % A.apart + 1) * A.G <= A.apart ? entry.y : 0;
    const int64_t first = at_part_at(A, slot, row, head), step = many ? (int64_t)all : A.part_stride;
    const int64_t first_own = (many ? A.own_at + at : A.group_splits * A.part_stride + first) - prefix * step;
    at_sum s = {-INFINITY, 0.0f, {0, 0, 0, 0}};
    for (int i = part; i < count; i += IN * LANES) {
        at_sum x[IN];
#pragma unroll
        for (int u = 0; u < IN; ++u) {
            x[u] = {-INFINITY, 0.0f, {0, 0, 0, 0}};
            const int p = i + u * LANES;
            if (p < count) {
                const int64_t from = p < prefix ? first + p * A.part_stride : first_own + p * step;
                const bl_v2f t = *bl_gc<bl_v2f>(A.part_ml + 2 * from);
                x[u].m = t[0], x[u].l = t[1], x[u].y = *bl_gc<bl_v4f>(A.many_part + from * D + d0);
            }
        }
#pragma unroll
        for (int u = 0; u < IN; ++u) s = at_add(s, x[u]);
    }
    if (LANES > 1) {
        if (d0 == 0) s_m[group] = s.m, s_l[group] = s.l;
        *(bl_v4f*)&s_y[group][d0] = s.y;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int j = 1; j < LANES; ++j) s = at_add(s, {s_m[j * ROWS + group], s_l[j * ROWS + group], *(const bl_v4f*)&s_y[j * ROWS + group][d0]});
    }
    if (count == 0 && !none) return;                          /* of no request, or done */
    const float inv = s.l == 0.0f ? 0.0f : bl_div_rn(1.0f, s.l);
    bl_v2u u = {bl_pack2_bf16(s.y[0] * inv, s.y[1] * inv), bl_pack2_bf16(s.y[2] * inv, s.y[3] * inv)};
    if (none) u = (bl_v2u){0x7fc07fc0u, 0x7fc07fc0u};         /* more queries than the launch was made for */
    *bl_g((bl_v2u*)(A.out + row * A.out_stride + head * D + d0)) = u;
}

/* ---- launches ---------------------------------------------------------------------------------------------------------- */

/* A batch without long runs of rows: at_few alone. */
template <int KIND, int D, bool WIDE, int ITEM>
__global__ __launch_bounds__(ITEM ? ITEM * BL_WAVE : AT_THREADS, 2) void bl_attn_few(at_args A) {
    constexpr size_t bytes = ITEM ? sizeof(at_meet_lds<D, ITEM ? ITEM : 1>) : sizeof(at_stream_lds<D>);
    __shared__ __attribute__((aligned(16))) uint8_t lds[bytes];
    at_few<KIND, D, WIDE, ITEM, true>(A, (int)blockIdx.x, lds);
}
/* One request, or groups of more heads than at_few has rows: at_many alone. */
template <int KIND, int D>
__global__ __launch_bounds__(AT_THREADS, 2) void bl_attn_many(at_args A) {
    __shared__ __attribute__((aligned(16))) at_many_lds<KIND, D> lds;
    at_many<KIND, D>(A, (int)blockIdx.x, lds);
}
/* Any batch, in one launch: the matrix cores' work first; what streams the cache fills the units as that ends. */
template <int KIND, int D, bool WIDE, int ITEM>
__global__ __launch_bounds__(AT_THREADS, 2) void bl_attn_any(at_args A, int many) {
    union lds_t {
        at_stream_lds<D> few;
        at_many_lds<KIND, D> many;
    };
    __shared__ __attribute__((aligned(16))) uint8_t lds[sizeof(lds_t)];
    if ((int)blockIdx.x < many) at_many<KIND, D>(A, (int)blockIdx.x, ((lds_t*)lds)->many);
    else at_few<KIND, D, WIDE, ITEM, false>(A, (int)blockIdx.x - many, lds);
}
/* Requests that share prefixes: workgroups of many rows of a request, of the prefixes, and of few rows behind them. */
template <int KIND, int D, bool WIDE, bool MANY>
__global__ __launch_bounds__(AT_THREADS, 2) void bl_attn_shared(at_args A, int prefix, int many) {
    union lds_t {
        at_meet_lds<D, AT_WAVES> few;
        at_prefix_lds<KIND, D> many;
    };
    __shared__ __attribute__((aligned(16))) uint8_t lds[sizeof(lds_t)];
    const int x = (int)blockIdx.x;
    if (MANY && x < many) at_many<KIND, D, AT_OWN>(A, x, ((lds_t*)lds)->many);
    else if (x < prefix + many) at_many<KIND, D, AT_PREFIX>(A, x - many, ((lds_t*)lds)->many);
    else at_few<KIND, D, WIDE, AT_WAVES, !MANY, true>(A, x - prefix - many, lds);
}
/* Partial results of both: `few` workgroups for those of at_few, turns x AT_STREAM_GROUPS, the others for a split. */
template <int D, bool MANY>
__global__ __launch_bounds__(AT_THREADS) void bl_attn_join(at_args A, int few) {
    __shared__ __attribute__((aligned(16))) at_join_lds<D> lds;
    const int x = (int)blockIdx.x;
    /* (sixteen partial results in flight are 122 registers: where a split's rows stand beside them, their loads need the waves more) */
    if (!MANY || x < few) at_few_join<D, MANY ? 4 : 16>(A, x % AT_STREAM_GROUPS, x / AT_STREAM_GROUPS, few / AT_STREAM_GROUPS, lds);
    else at_many_join<D>(A, x - few);
}

/* ---- host ------------------------------------------------------------------------------------------------------------- */

struct at_plan {
    bool few, many;
    int items;                     /* workgroups, an item each; 0: streams */
    int splits, row_tiles, skip, rows;
    size_t few_bytes, bytes;
};

static bl_status at_check(const bl_attn_desc* a) {
    if (!a) return BL_ERR_NULL;
    if (const bl_status rc = bl_kv_cache_check(&a->cache)) return rc;
    if (!a->q || !a->q_start || !a->seq_len || !a->table || !a->out) return BL_ERR_NULL;
    const int64_t most = (int64_t)1 << 40, width = (int64_t)a->n_q * a->cache.head_dim;
    if (a->B < 1 || a->B > BL_KV_MAX_REQUESTS || a->T < 1 || a->T > BL_MAX_DIM || a->n_q < 1 || a->n_q > 65535 || a->n_q % a->cache.n_kv ||
        a->max_blocks < 1 || (int64_t)a->max_blocks * a->cache.block > ((int64_t)1 << 30) || a->table_stride < a->max_blocks || a->table_stride > most ||
        a->max_q < 1 || a->max_len < 0 || a->window < 0 || a->q_stride < width || a->q_stride > most || a->out_stride < width || a->out_stride > most ||
        a->T * (a->n_q / a->cache.n_kv) > ((int64_t)1 << 30) || a->B * a->cache.n_kv * ((int64_t)a->max_blocks * a->cache.block / AT_TILE + 2) > ((int64_t)1 << 30))
        return BL_ERR_SHAPE;
    if (!(a->softmax_scale > 0.0f) || a->softmax_scale > 3e38f) return BL_ERR_VALUE;
    if (!bl_aligned(a->q, 16) || !bl_aligned(a->out, 16) || a->q_stride % 8 || a->out_stride % 8 || !bl_aligned(a->q_start, 4) ||
        !bl_aligned(a->seq_len, 4) || !bl_aligned(a->table, 4))
        return BL_ERR_ALIGN;
    return BL_OK;
}

static at_plan at_make_plan(const bl_attn_desc* a) {
    at_plan p;
    const int G = a->n_q / a->cache.n_kv, D = a->cache.head_dim;
    const int64_t rows = (int64_t)(a->max_q < a->T ? a->max_q : a->T) * G;
    p.many = rows > AT_FEW;
    p.few = G <= AT_FEW && !(p.many && a->B == 1);            /* (one request: of one kind or the other) */
    /* Tokens that the rows of a workgroup see (the length alone under a window of 1000, 16 requests of 4 queries over 8000: 23.5 us, so 12.5;
     * 64 queries, a window of 500: 22.5 and 19.7). */
    int64_t tokens = a->max_len > 0 ? a->max_len : (int64_t)a->max_blocks * a->cache.block;
    const int64_t wide = (int64_t)a->window + (a->max_q < AT_MANY ? a->max_q : AT_MANY);
    if (a->window && tokens > wide) tokens = wide;
    /* An item a workgroup, without a join, while its tokens are few, more where there are items for every unit.  Time in us as items and as
     * streams, equal lengths / spread over a quarter to the whole:
     * heads of 128: 5 items (of one request) of 512 tokens 8 and 11, 1024 11 and 11, 2048 18 and 11; 160 of 1500 17 and 21 / 16 and 20;
     *   320 of 1500 32 and 32 / 26 and 27, of 2048 41 and 37 / 34 and 28; 1280 of 2048 106 and 120 / 74 and 79, of 4096 140 and 136;
     * heads of 64: 8 of 1024 7.7 and 11.8, 2048 10 and 11.5, 4096 16 and 12; 128 of 4096 17.2 and 19.4 / 16.5 and 17.1; 1024 of 4096 83 and 89 / 54 and 58.
     * Heads of 64 where there is an item a unit at most: eight waves, which have more loads on their way (128 of 2048 13.0 -> 11.0; 512 of 512 12.8 -> 14.6).
     * Beside many rows (four waves then), heads of 64, streams and items: 4 requests over 300 15.2 and 13.1; 16 over 1000 33 and 29, 64 28 and 26, 256 50 and 39;
     *   256 over 2000 79 and 67; 32 over 2000 25.4 and 26.4; 6 over 1802 23.8 and 25.2; 16 over 2500 26.4 and 26.5; but 64 over 3500 60 and 58, 256 over 4000
     *   140 and 127, where five eighths leave them to the streams.  Heads of 128: the same within 1 % over all of these.
     * Heads of 128 gain nothing from them (18 -> 19.5): four lanes that stand together read four lines of K, and a unit takes a line a clock. */
    const int64_t items = a->B * a->cache.n_kv;
    const int64_t alone = D == 128 ? items >= 1024 ? 2048 : items >= 128 ? 1536 : 1024 : items >= 128 ? 4096 : 2048;
    const int64_t most = D == 64 && p.many ? alone * 5 / 8 : alone;
    p.items = p.few && tokens <= most ? (int)items : 0;
    const int64_t part = a->T < a->B ? a->T : a->B;           /* requests with rows */
    p.row_tiles = (int)(a->T * G / AT_MANY + part);
    p.splits = 1;
    if (p.many) {
        /* pieces until the workgroups fill the chip twice over, of four tiles at least (64 queries over 1000 tokens: of eight 33.5 us, of four
         * 19.9, of two 17.4; over 4000: 27.1, 23.1 and 27.1) */
        const int64_t items = (int64_t)((a->T * G + AT_MANY - 1) / AT_MANY) * a->cache.n_kv;
        int64_t s = items < 512 ? 512 / items : 1;
        const int64_t by_len = tokens / (4 * AT_TILE);
        s = s > by_len ? by_len : s;
        p.splits = s < 1 ? 1 : s > 64 ? 64 : (int)s;
    }
    p.skip = p.few ? (int)((a->B + 15) / 16 * 64) : 0;
    /* (items leave no partial results: theirs is an address, 256 bytes for every 16 requests instead of 34 MB with heads of 128) */
    p.few_bytes = p.few ? ((p.items ? 0 : (size_t)AT_STREAMS * 2 * AT_FEW * (D + 2)) + p.skip) * sizeof(float) : 0;
    p.rows = (int)(rows < AT_FEW ? rows : AT_FEW);
    p.bytes = p.few_bytes + (p.splits > 1 ? (size_t)p.splits * a->T * a->n_q * (D + 2) * sizeof(float) : 0);
    return p;
}

extern "C" size_t bl_attn_workspace_bytes(const bl_attn_desc* a) {
    return at_check(a) == BL_OK ? at_make_plan(a).bytes : 0;
}

static at_args at_make_args(const bl_attn_desc* a) {
    const bl_kv_cache& c = a->cache;
    at_args A = {};
    A.k = (const uint8_t*)c.k, A.v = (const uint8_t*)c.v, A.k_scale = c.k_scale, A.v_scale = c.v_scale;
    A.q = a->q, A.q_start = a->q_start, A.seq_len = a->seq_len, A.table = a->table, A.out = a->out;
    A.k_units = (uint32_t)(c.k_stride / 16), A.v_units = (uint32_t)(c.v_stride / 16), A.scale_stride = c.scale_stride;
    A.q_stride = a->q_stride, A.out_stride = a->out_stride, A.table_stride = a->table_stride;
    A.n_blocks = (int)c.n_blocks, A.n_kv = c.n_kv, A.G = a->n_q / c.n_kv, A.n_q = a->n_q, A.B = (int)a->B, A.T = (int)a->T;
    A.shift = bl_log2(c.block), A.max_tokens = a->max_blocks * c.block, A.window = a->window < 1 << 30 ? a->window : 1 << 30;
    A.factor = a->softmax_scale * 1.44269504f;
    return A;
}

template <int KIND, int D, bool WIDE>
static void at_launch(at_args A, const at_plan& p, const bl_attn_desc* a, hipStream_t st) {
    A.part = (float*)a->workspace;
    A.many_part = A.part + p.few_bytes / sizeof(float);
    const int few = !p.few ? 0 : p.items ? p.items : AT_STREAM_GROUPS;
    if (p.many) {
        const int many = p.row_tiles * A.n_kv * p.splits;
        if (few && p.items) bl_attn_any<KIND, D, WIDE, AT_WAVES><<<(unsigned)(many + few), AT_THREADS, 0, st>>>(A, many);
        else if (few) bl_attn_any<KIND, D, WIDE, 0><<<(unsigned)(many + few), AT_THREADS, 0, st>>>(A, many);
        else bl_attn_many<KIND, D><<<(unsigned)many, AT_THREADS, 0, st>>>(A);
    } else {
        if (p.items) {
            if (D == 64 && p.items <= 256) bl_attn_few<KIND, D, WIDE, D == 64 ? 8 : 4><<<(unsigned)p.items, 8 * BL_WAVE, 0, st>>>(A);
            else bl_attn_few<KIND, D, WIDE, 4><<<(unsigned)p.items, 4 * BL_WAVE, 0, st>>>(A);
            return;
        }
        bl_attn_few<KIND, D, WIDE, 0><<<(unsigned)few, AT_THREADS, 0, st>>>(A);
    }
    const int64_t rows = (int64_t)A.T * A.n_q, per = AT_THREADS / (D / 4);
    const int few_join = p.few && !p.items ? AT_STREAM_GROUPS * ((p.rows + 256 / D - 1) / (256 / D)) : 0;      /* (D / 4 lanes a row of a wave) */
    const int64_t join = few_join + (p.splits > 1 ? (rows + per - 1) / per : 0);
    if (p.splits > 1) bl_attn_join<D, true><<<(unsigned)join, AT_THREADS, 0, st>>>(A, few_join);
    else if (join) bl_attn_join<D, false><<<(unsigned)join, AT_THREADS, 0, st>>>(A, few_join);
}

extern "C" bl_status bl_attn_kv8(const bl_attn_desc* a, bl_stream s) {
    if (const bl_status rc = at_check(a)) return rc;
    const at_plan p = at_make_plan(a);
    if (p.bytes && !a->workspace) return BL_ERR_WORKSPACE;
    if (!bl_aligned(a->workspace, 256)) return BL_ERR_ALIGN;
    const bl_kv_cache& c = a->cache;
    if ((int64_t)p.row_tiles * c.n_kv * p.splits + p.items > 0x7fff0000) return BL_ERR_SHAPE;
    at_args A = at_make_args(a);
    A.few_rows = p.few ? AT_FEW : 0, A.splits = p.splits, A.part_skip = p.skip;
    const hipStream_t st = (hipStream_t)s;
#define AT(K, D) (c.block == 128 ? at_launch<K, D, true>(A, p, a, st) : at_launch<K, D, false>(A, p, a, st))
    if (c.kind == BL_KV_INT8) c.head_dim == 128 ? AT(BL_KV_INT8, 128) : AT(BL_KV_INT8, 64);
    else c.head_dim == 128 ? AT(BL_KV_E4M3, 128) : AT(BL_KV_E4M3, 64);
#undef AT
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}

/* ---- shared prefixes, host ------------------------------------------------------------------------------------------------ */

struct at_shared_plan {
    bool few, many, by_request;
    int group_splits, few_splits, many_splits, apart;
    int64_t prefix_tiles, many_tiles, part_stride, own_at, parts;
    size_t pieces, bytes;          /* of the rows' entries in front, and in all */
};

static bl_status at_check_shared(const bl_attn_shared_desc* a) {
    if (!a) return BL_ERR_NULL;
    if (const bl_status rc = at_check(&a->attn)) return rc;
    if (!a->group || !a->shared_blocks || !a->shared_table) return BL_ERR_NULL;
    if (a->n_groups < 1 || a->n_groups > BL_KV_MAX_REQUESTS || a->max_shared < 1 || (int64_t)a->max_shared * a->attn.cache.block > ((int64_t)1 << 30) ||
        a->shared_stride < a->max_shared || a->shared_stride > ((int64_t)1 << 40) || a->max_own < 0)
        return BL_ERR_SHAPE;
    if (!bl_aligned(a->group, 4) || !bl_aligned(a->shared_blocks, 4) || !bl_aligned(a->shared_table, 4)) return BL_ERR_ALIGN;
    return BL_OK;
}

/* Whether bl_attn_kv8's kernels do it, which read the prefix once a request: where contexts are short enough for a workgroup an item, which leaves nothing
 * to join, or there is little to read at all.  us of these kernels and of those, all requests behind one prefix, up to 300 tokens of their own:
 *   20 + 5 heads of 128, prefix 500: 2 to 64 requests 11 to 18 and 9 to 14 (four queries each 12 to 23 and 9 to 15); 2000: 2, 4, 8, 16, 64 requests 12.8, 13.2, 14.0, 15.2,
 *     22.2 and 11.4, 11.7, 14.6, 18.6, 34.7; 8000: 17.1 to 32 and 17.6 to 83; 30000: 26 to 33 (16 requests) and 27 to 107;
 *   32 + 8 heads of 64, 2000: 2 to 64 requests 11.5 to 17 and 10 to 15; 3000: 16, 64 requests 14.2, 20 and 11, 19 to 21, 48 of four queries, one group and five, 29 and 34 and 18 to 21; 3500:
 *     14.7, 20 and 12, 21 to 23; 4096: 15, 21.7 and 19, 37; 8000: 15.1 to 27.7 and 13.9 to 60; 16 + 1 of 128, 2000: 12.4 to 20.4 and 11.6 to 22.8. */
static bool at_shared_apart(const bl_attn_shared_desc* s) {
    const bl_attn_desc* a = &s->attn;
    const int64_t tokens = a->max_len > 0 ? a->max_len : (int64_t)a->max_blocks * a->cache.block;
    return at_make_plan(a).items || (tokens < 4096 && a->B * a->cache.n_kv * tokens < 65536);
}

static at_shared_plan at_make_shared_plan(const bl_attn_shared_desc* s) {
    const bl_attn_desc* a = &s->attn;
    at_shared_plan p;
    const int G = a->n_q / a->cache.n_kv, D = a->cache.head_dim;
    p.many = (int64_t)(a->max_q < a->T ? a->max_q : a->T) * G > AT_FEW, p.few = G <= AT_FEW;
    const int64_t tiles = (a->T * G + AT_MANY - 1) / AT_MANY, part = a->T < a->B ? a->T : a->B, groups = s->n_groups < part ? s->n_groups : part;
    int64_t tokens = a->max_len > 0 ? a->max_len : (int64_t)a->max_blocks * a->cache.block, own = s->max_own > 0 ? s->max_own : tokens;
    const int64_t wide = (int64_t)a->window + (a->max_q < AT_MANY ? a->max_q : AT_MANY);
    if (a->window && tokens > wide) tokens = wide;
    if (a->window && own > wide) own = wide;
    /* Pieces of `items` items of `tokens`: until there are 512 workgroups while a piece has `deep` tiles, 256 while it has four, 128 while all but the last have `each`. */
    auto pieces = [](int64_t items, int64_t tokens, int64_t deep, int64_t each, int64_t most) -> int {
        auto until = [&](int64_t groups, int64_t pieces) { return std::min(groups / items, pieces); };
        const int64_t n = std::max(std::max(until(512, tokens / (deep * AT_TILE)), until(256, tokens / (4 * AT_TILE))), until(128, (tokens + each * AT_TILE - 1) / (each * AT_TILE)));
        return (int)(n < 1 ? 1 : n < most ? n : most);
    };
    /* Where a request may fill tiles of at_many by itself, which read the prefix from the caches then, all of more than AT_FEW rows are apart; else they are of
     * their groups.  us of this and of the other, 20 + 5 heads: 8 chunks of 300 beside 16 decoding requests behind 4096 tokens 124 and 135, 4 of 300 beside 60
     * behind 8000 110 and 127; 30 queries of each of 16 requests behind 32000 216 and 293, 20 of 24 behind 4096 59 and 68.  What it costs: requests of 17 to 127 rows beside a prompt read the
     * prefix each for itself then, 60 of five queries (20 rows) beside one chunk of 300 behind 8000 and 32000 tokens 217 and 750, bl_attn_kv8 208 and 692, without the chunk 71 and 149. */
    const bool prompts = p.many && (int64_t)a->max_q * G >= AT_MANY;
    p.apart = prompts ? AT_FEW + 1 : AT_MANY;
    const int64_t most = a->T * G < part * (p.apart - 1) ? a->T * G : part * (p.apart - 1);            /* rows that groups can have */
    p.prefix_tiles = most / AT_MANY + groups;
    /* (64 requests behind 4096 tokens, 256 with pieces of three tiles 33.0, of four 28.5.  Heads of 128, two workgroups a unit: the second pays for itself where it has sixteen tiles.  us so and with 512 of four tiles: 64 requests behind 16000 tokens, 5, 8
     * and 1 kv heads 38, 48, 37 and 47, 55, 40, 128 behind 8000 42, 56, 39 and 51, 66, 43; 512 and 256 where there are sixteen: 16 behind 65536, 8 kv heads, 56 and 67.
     * Not where one piece is half of the 256 (200 requests, 30 of them with 30 queries, behind 2000, 170 items: one piece 105, three 77), or prompts are on the units too (four of
     * 300 tokens beside 60 behind 8000: 116 and 107).  Heads of 64, three a unit: 64 behind 16000 34.5 with 512, 38 with 256) */
    const int64_t items = (most + AT_MANY - 1) / AT_MANY * a->cache.n_kv;
    p.group_splits = pieces(items, (int64_t)s->max_shared * a->cache.block, D == 128 && items <= 128 && !prompts ? 16 : 4, 1, 64);
    p.few_splits = p.few ? pieces(part * a->cache.n_kv, own, 4, 4, 32) : 0;
    /* (prompts read the prefix too: two of 600 over 32000 tokens beside 14 of one, cut by their own tokens 790 us, by all 370) */
    p.many_splits = p.many ? pieces(tiles * a->cache.n_kv, prompts ? tokens : own, 4, 4, 32) : 0;
    p.many_tiles = p.many ? a->T * G / AT_MANY + part : 0;
    p.pieces = ((size_t)a->T * sizeof(int2) + 255) / 256 * 256;
    p.by_request = a->B * a->cache.n_kv * p.apart < a->T * a->n_q;
    p.part_stride = p.by_request ? a->B * a->cache.n_kv * p.apart : a->T * a->n_q;
    p.own_at = (p.group_splits + p.few_splits) * p.part_stride, p.parts = p.own_at + p.many_splits * a->T * a->n_q;
    p.bytes = p.pieces + (size_t)p.parts * (D + 2) * sizeof(float);
    return p;
}

extern "C" size_t bl_attn_shared_workspace_bytes(const bl_attn_shared_desc* a) {
    return at_check_shared(a) != BL_OK ? 0 : at_shared_apart(a) ? at_make_plan(&a->attn).bytes : at_make_shared_plan(a).bytes;
}

/* Workgroups up to which the join takes four groups of threads a row (24 requests, 80 rows: 38.6 us, with one 40.7; 1467 rows: 147.7, so 134.5). */
#define AT_JOIN_LANES 4096
template <int KIND, int D, bool WIDE>
static void at_shared_launch(const at_args& A, const at_shared_plan& p, hipStream_t st) {
    const int prefix = (int)(p.prefix_tiles * A.n_kv * p.group_splits), many = (int)(p.many_tiles * A.n_kv * p.many_splits);
    const int few = p.few ? A.B * A.n_kv * p.few_splits : 0;
    if (p.many) bl_attn_shared<KIND, D, WIDE, true><<<(unsigned)(prefix + many + few), AT_THREADS, 0, st>>>(A, prefix, many);
    else bl_attn_shared<KIND, D, WIDE, false><<<(unsigned)(prefix + few), AT_THREADS, 0, st>>>(A, prefix, 0);
    const int64_t rows = (int64_t)A.T * A.n_q, per = AT_THREADS / (D / 4);
    if (p.group_splits + (p.few_splits > p.many_splits ? p.few_splits : p.many_splits) <= 4 || rows * 4 / per > AT_JOIN_LANES) bl_attn_shared_join<D, 1><<<(unsigned)((rows + per - 1) / per), AT_THREADS, 0, st>>>(A);
    else bl_attn_shared_join<D, 4><<<(unsigned)((rows * 4 + per - 1) / per), AT_THREADS, 0, st>>>(A);
}

extern "C" bl_status bl_attn_kv8_shared(const bl_attn_shared_desc* s, bl_stream stream) {
    if (const bl_status rc = at_check_shared(s)) return rc;
    const bl_attn_desc* a = &s->attn;
    if (at_shared_apart(s)) return bl_attn_kv8(a, stream);
    const at_shared_plan p = at_make_shared_plan(s);
    if (!a->workspace) return BL_ERR_WORKSPACE;
    if (!bl_aligned(a->workspace, 256)) return BL_ERR_ALIGN;
    const bl_kv_cache& c = a->cache;
    /* (a launch counts its threads in 32 bits) */
    if (c.n_kv * (p.prefix_tiles * p.group_splits + p.many_tiles * p.many_splits + a->B * p.few_splits) >= 1 << 24 || a->T * a->n_q * (c.head_dim / 4) >= (int64_t)1 << 32)
        return BL_ERR_SHAPE;
    at_args A = at_make_args(a);
    A.few_rows = p.few ? AT_FEW : 0, A.group_splits = p.group_splits, A.few_splits = p.few_splits, A.many_splits = p.many_splits;
    A.group = s->group, A.shared_blocks = s->shared_blocks, A.shared_table = s->shared_table, A.shared_stride = s->shared_stride;
    A.n_groups = (int)s->n_groups, A.max_shared = s->max_shared;
    A.pieces = (int2*)a->workspace, A.many_part = (float*)((char*)a->workspace + p.pieces), A.part_ml = A.many_part + p.parts * c.head_dim;
    A.part_stride = p.part_stride, A.own_at = p.own_at, A.by_request = p.by_request, A.apart = p.apart;
    const hipStream_t st = (hipStream_t)stream;
#define AT(K, D) (c.block == 128 ? at_shared_launch<K, D, true>(A, p, st) : at_shared_launch<K, D, false>(A, p, st))
    if (c.kind == BL_KV_INT8) c.head_dim == 128 ? AT(BL_KV_INT8, 128) : AT(BL_KV_INT8, 64);
    else c.head_dim == 128 ? AT(BL_KV_E4M3, 128) : AT(BL_KV_E4M3, 64);
#undef AT
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}
