/* Key/value cache of 8-bit codes: the block tables of a step and the rotary append of its tokens (bitlinear.h). */
#include "bl_device.h"
#include "bl_kv.h"

/* ---- block tables and slot maps ---------------------------------------------------------------------------------- */

/* Blocks that a request's own thread takes; more are copied by waves.  256 requests of one / two / three / four new blocks each: by the thread 9.5 / 9.6 /
 * 10.0 / 10.1 us, by waves 13.8 / 13.8 / 14.1 / 13.9; 8 requests 3.3 / 3.5 / 4.0 / 4.2 and 4.2 / 4.3 / 4.5 / 4.6.  (Three and four would gain, left as it is.) */
#define TAB_OWN 2
/* Rows whose slots the table kernel writes itself; a second launch does more.  8, 64 and 400 requests, itself against the launch: some 2000 rows
 * 6.2, 7.1, 7.5 us against 7.6, 8.8, 10.0; 4500 rows 7.1, 8.7, 9.3 against 7.5, 9.0, 10.0; 9000 rows 9.2, 12.9, 12.6 against 7.5, 10.2, 10.1. */
#define TAB_ROWS_INSIDE 4096

template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t tab_moved(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, ROWS == 0xf);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, ROWS == 0xf);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
/* Sum of v over the threads in front of this one, and over all (in *total).  s: a value a wave, reused after a barrier. */
template <int THREADS>
__device__ __forceinline__ int64_t tab_scan(int64_t v, int64_t* s, int64_t* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t x = v;
    x += tab_moved<0x111, 0xf>(x);               /* row_shr 1, 2, 4, 8 */
    x += tab_moved<0x112, 0xf>(x);
    x += tab_moved<0x114, 0xf>(x);
    x += tab_moved<0x118, 0xf>(x);
    x += tab_moved<0x142, 0xa>(x);               /* row_bcast 15 into rows 1 and 3, 31 into 2 and 3 */
    x += tab_moved<0x143, 0xc>(x);
    __syncthreads();
    if (lane == 63) s[w] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / BL_WAVE; ++i) {
        const int64_t t = s[i];
        before += i < w ? t : 0;
        all += t;
    }
    *total = all;
    return before + x - v;
}
/* Adds this wave's requests r of which `has` holds to a list in LDS. */
__device__ __forceinline__ void tab_list(bool has, int r, int* list, int* count) {
    const uint64_t m = __ballot(has);
    if (!m) return;
    const int lane = threadIdx.x & 63;
    int at = 0;
    if (lane == 0) at = atomicAdd(count, __builtin_popcountll(m));
    at = __builtin_amdgcn_readlane(at, 0) + __builtin_popcountll(m & (((uint64_t)1 << lane) - 1));
    if (has) list[at] = r;
}

/* The n[r] entries of every listed request r from from(r) (STEP -1: downwards) to to(r): a wave has four requests at a time, IN / 4 entries of
 * each a lane in flight.  256 requests of up to 4096 tokens, a ninth of which ends: 5.8 us, one request a wave at a time 9.8 (1024: 8.4 and 13.2); where all
 * that end have 512 blocks, 57 of 512 requests, the other way round: 10.1 and 8.3. */
template <int WAVES, int IN, int STEP, typename F, typename G>
__device__ __forceinline__ void tab_copy(const int* list, int count, const int* n, F from, G to) {
    constexpr int MANY = 4, EACH = IN / MANY;
    const int lane = threadIdx.x & 63;
    for (int k = threadIdx.x >> 6; k < count; k += MANY * WAVES) {
        const int32_t* src[MANY];
        int32_t* dst[MANY];
        int have[MANY], most = 0;
#pragma unroll
        for (int i = 0; i < MANY; ++i) {
            const bool there = k + i * WAVES < count;
            const int r = list[there ? k + i * WAVES : k];
            have[i] = there ? n[r] : 0, src[i] = from(r), dst[i] = to(r);
            most = have[i] > most ? have[i] : most;
        }
        for (int j = lane; j < most; j += EACH * 64) {
            int v[MANY][EACH];
#pragma unroll
            for (int i = 0; i < MANY; ++i)
#pragma unroll
                for (int u = 0; u < EACH; ++u)
                    if (j + 64 * u < have[i]) v[i][u] = src[i][STEP * (j + 64 * u)];
#pragma unroll
            for (int i = 0; i < MANY; ++i)
#pragma unroll
                for (int u = 0; u < EACH; ++u)
                    if (j + 64 * u < have[i]) dst[i][j + 64 * u] = v[i][u];
        }
    }
}

/* Position and slot of row t of the batch: its request by bisection in the B + 1 ascending first rows. */
__device__ __forceinline__ void tab_row(int64_t t, int B, const int* q_start, const int* start, const int32_t* table, int64_t table_stride,
                                        int shift, int32_t* positions, int32_t* slots) {
    int pos = 0, slot = -1;
    if (t < q_start[B]) {
        int lo = 0, hi = B;                      /* q_start[lo] <= t < q_start[hi] */
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (q_start[mid] <= t) lo = mid;
            else hi = mid;
        }
        if (start[lo] >= 0) {
            pos = start[lo] + (int)(t - q_start[lo]);
            const uint32_t block = (uint32_t)table[lo * table_stride + (pos >> shift)];
            slot = block < 0x80000000u >> shift ? (int)((block << shift) + (uint32_t)(pos & ((1 << shift) - 1))) : -2;    /* (no block: not another's slot) */
        }
    }
    positions[t] = pos;
    slots[t] = slot;
}

struct tab_args {
    bl_kv_batch b;
    int shift, max_new;
};

/* One workgroup: a handful of requests, or a few thousand, is latency and not work.  Three sums over the requests (rows
 * and returned blocks, then demand, which needs them), the copies between stack and table by waves (one or two blocks by the
 * request's thread), then the rows.  A thread holds PER consecutive requests where there are more than threads.
 * Bound by the launch and three dependent reads (lengths, stack, table): 8 requests 3.9 us, 512 with 33 thousand rows, 57 of them
 * ending, 9 and 4 for the rows' own kernel.  Above 1024 requests (PER 4: 30 vector registers spilled) 1025 take 12.7 us, 2048 17.2, 4096 30. */
template <int THREADS, int PER, bool LIMIT>
__global__ __launch_bounds__(THREADS) void bl_kv_tables_kernel(tab_args A) {
    const bl_kv_batch& b = A.b;
    constexpr int MOST = THREADS * PER, WAVES = THREADS / BL_WAVE, IN = 8;
    __shared__ int64_t s_sum[WAVES];
    __shared__ int s_start[MOST], s_row[MOST + 1], s_list[MOST], s_from[MOST], s_n[MOST];
    __shared__ int s_taken, s_bad, s_back, s_want;
    const int tid = threadIdx.x, B = (int)b.B, shift = A.shift, bs1 = (1 << shift) - 1;
    const int per = PER == 1 ? 1 : (B + THREADS - 1) / THREADS;
    if (tid == 0) s_taken = s_bad = s_back = s_want = 0;
    const int64_t cap = b.free_cap;
    int64_t there = b.free_count[0];
    int old[PER], n[PER];
    int64_t rows = 0, back = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = tid * per + i;
        old[i] = n[i] = 0;
        if (i < per && r < B) {
            const int64_t most = (int64_t)b.max_blocks << shift;
            const int64_t L = b.seq_len[r];
            old[i] = (int)(L < 0 ? 0 : L > most ? most : L);
            n[i] = b.new_len[r];
        }
        if (n[i] < 0) back += ((int64_t)old[i] + bs1) >> shift;
        else rows += n[i];
    }
    there = there < 0 ? 0 : there > cap ? cap : there;
    int64_t all_rows, all_back;
    int64_t row = tab_scan<THREADS>(rows, s_sum, &all_rows);
    int64_t at = there + tab_scan<THREADS>(back, s_sum, &all_back);
    if (all_back) {
        /* ended requests: their blocks to the stack */
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i >= per) break;
            const int r = tid * per + i, have = n[i] < 0 ? (int)(((int64_t)old[i] + bs1) >> shift) : 0;
            if (have > 0 && at + have > cap) atomicAdd(&s_bad, 1);
            if (have > 0) s_from[r] = (int)(at < cap ? at : cap), s_n[r] = at < cap ? (int)(cap - at < have ? cap - at : have) : 0;
            tab_list(have > 0, r, s_list, &s_back);
            at += have;
        }
        __syncthreads();
        tab_copy<WAVES, IN, 1>(s_list, s_back, s_n, [&](int r) { return b.table + r * b.table_stride; }, [&](int r) { return b.free_list + s_from[r]; });
    }
    there = there + all_back > cap ? cap : there + all_back;
    /* demand */
    int64_t want = 0, row_i = row;
    int w_i[PER];
    bool fits[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int64_t need = ((int64_t)old[i] + (n[i] > 0 ? n[i] : 0) + bs1) >> shift;
        row_i += n[i] > 0 ? n[i] : 0;
        fits[i] = n[i] >= 0 && (!LIMIT || n[i] <= A.max_new) && need <= b.max_blocks && row_i <= b.rows;
        w_i[i] = fits[i] ? (int)(need - (((int64_t)old[i] + bs1) >> shift)) : 0;
        want += w_i[i];
    }
    int64_t all_want;
    int64_t upto = tab_scan<THREADS>(want, s_sum, &all_want);       /* (its barriers: the stack is whole behind them) */
    row_i = row;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        const int r = tid * per + i;
        const bool live = r < B;
        const int64_t before = upto;
        upto += w_i[i];
        const bool ok = live && fits[i] && (w_i[i] == 0 || upto <= there), takes = ok && w_i[i] > 0;
        if (live && n[i] >= 0 && !ok) atomicAdd(&s_bad, 1);
        if (takes) {
            const int has = (int)(((int64_t)old[i] + bs1) >> shift);
            atomicMax(&s_taken, (int)upto);
            s_from[r] = (int)(there - 1 - before), s_n[r] = w_i[i], s_start[r] = has;       /* (for now: the blocks that it has) */
            if (w_i[i] <= TAB_OWN) {
                const int32_t* from = b.free_list + (there - 1 - before);
                int32_t* to = b.table + r * b.table_stride + has;
                const int v = from[0];
                if (w_i[i] > 1) to[1] = from[-1];
                to[0] = v;
            }
        }
        tab_list(takes && w_i[i] > TAB_OWN, r, s_list, &s_want);
        row_i += n[i] > 0 ? n[i] : 0;
    }
    if (all_want) {
        __syncthreads();
        tab_copy<WAVES, IN, -1>(s_list, s_want, s_n, [&](int r) { return b.free_list + s_from[r]; }, [&](int r) { return b.table + r * b.table_stride + s_start[r]; });
        __syncthreads();
    }
    upto -= want, row_i = row;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        const int r = tid * per + i;
        upto += w_i[i];
        const bool ok = fits[i] && (w_i[i] == 0 || upto <= there);
        if (r < B) {
            const int first = (int)(row_i < b.rows ? row_i : b.rows), st = ok ? old[i] : -1;
            s_start[r] = b.start[r] = st;
            s_row[r] = b.q_start[r] = first;
            b.seq_len_out[r] = n[i] < 0 ? 0 : ok ? old[i] + n[i] : old[i];
        }
        row_i += n[i] > 0 ? n[i] : 0;
    }
    if (tid == 0) s_row[B] = b.q_start[B] = (int)(all_rows < b.rows ? all_rows : b.rows);
    __syncthreads();
    if (tid == 0) {
        b.free_count_out[0] = (int)there - s_taken;
        b.bad[0] = s_bad;
    }
    if (b.rows <= TAB_ROWS_INSIDE)
        for (int64_t t = tid; t < b.rows; t += THREADS) tab_row(t, B, s_row, s_start, b.table, b.table_stride, shift, b.positions, b.slots);
}

/* The rows of a large batch, behind the table kernel: one thread a row. */
__global__ __launch_bounds__(256) void bl_kv_slots_kernel(tab_args A) {
    const bl_kv_batch& b = A.b;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < b.rows) tab_row(t, (int)b.B, b.q_start, b.start, b.table, b.table_stride, A.shift, b.positions, b.slots);
}

/* LIMIT: with a most of new tokens a request (a kernel of its own: above 1024 requests the comparison costs the others 1.2 us). */
template <bool LIMIT>
static bl_status tab_launch(const bl_kv_batch* b, int max_new, bl_stream s) {
    if (!b->seq_len || !b->new_len || !b->free_count || !b->table || (!b->free_list && b->free_cap) || !b->seq_len_out || !b->free_count_out || !b->start ||
        !b->q_start || !b->positions || !b->slots || !b->bad)
        return BL_ERR_NULL;
    if (!bl_kv_block_ok(b->block) || b->B < 1 || b->B > BL_KV_MAX_REQUESTS || b->rows < 1 || b->rows > BL_MAX_DIM || b->max_blocks < 1 ||
        (int64_t)b->max_blocks * b->block > 0x7fffffff || b->table_stride < b->max_blocks || b->table_stride > ((int64_t)1 << 40) || b->free_cap < 0 ||
        b->free_cap > 0x7fffffff)
        return BL_ERR_SHAPE;
    const void* p[] = {b->seq_len, b->new_len, b->free_count, b->table, b->free_list, b->seq_len_out, b->free_count_out, b->start, b->q_start, b->positions, b->slots, b->bad};
    for (const void* q : p)
        if (!bl_aligned(q, 4)) return BL_ERR_ALIGN;
    tab_args A = {*b, bl_log2(b->block), max_new};
    /* A small step's barriers are those of four waves instead of sixteen: 1, 64 and 256 decoding requests 2.8, 4.4 and 5.8 us, with sixteen 4.3, 5.9 and
     * 6.5; beside a chunk of 1024 rows the rows' loop has the more of it: 64 and 256 requests 7.6 and 9.4 us with four, 7.2 and 7.8 with sixteen. */
    if (b->B <= 256 && b->rows <= 1024) bl_kv_tables_kernel<256, 1, LIMIT><<<1, 256, 0, (hipStream_t)s>>>(A);
    else if (b->B <= 1024) bl_kv_tables_kernel<1024, 1, LIMIT><<<1, 1024, 0, (hipStream_t)s>>>(A);
    else bl_kv_tables_kernel<1024, BL_KV_MAX_REQUESTS / 1024, LIMIT><<<1, 1024, 0, (hipStream_t)s>>>(A);
    if (b->rows > TAB_ROWS_INSIDE) bl_kv_slots_kernel<<<(unsigned)((b->rows + 255) / 256), 256, 0, (hipStream_t)s>>>(A);
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}

extern "C" bl_status bl_kv_tables(const bl_kv_batch* b, bl_stream s) { return b ? tab_launch<false>(b, 0, s) : BL_ERR_NULL; }

extern "C" bl_status bl_kv_tables_limited(const bl_kv_limited_batch* b, bl_stream s) {
    if (!b) return BL_ERR_NULL;
    if (b->max_new < 1) return BL_ERR_SHAPE;
    return tab_launch<true>(&b->batch, b->max_new < 0x7fffffff ? (int)b->max_new : 0x7fffffff, s);
}

/* ---- rotary append ----------------------------------------------------------------------------------------------- */

#define APP_THREADS 256

struct app_args {
    bl_kv_tokens t;
    int shift, window, windows;            /* log2(block); rows of a K/V workgroup, and how many such there are */
};

typedef uint32_t app_v4u __attribute__((ext_vector_type(4)));
/* Four consecutive values of a row. */
template <int SRC>
__device__ __forceinline__ void app_load4(const void* row, int64_t i, float (&v)[4]) {
    if (SRC == BL_KV_FROM_F32) {
        const bl_v4f x = *bl_gc<bl_v4f>((const float*)row + i);
        v[0] = x[0], v[1] = x[1], v[2] = x[2], v[3] = x[3];
    } else {
        const bl_v2u x = *bl_gc<bl_v2u>((const uint16_t*)row + i);
        v[0] = bl_bf16_to_f32(x[0] & 0xffff), v[1] = __uint_as_float(x[0] & 0xffff0000u);
        v[2] = bl_bf16_to_f32(x[1] & 0xffff), v[3] = __uint_as_float(x[1] & 0xffff0000u);
    }
}
template <int SRC>
__device__ __forceinline__ const void* app_row(const app_args& A, int64_t t) {
    return SRC == BL_KV_FROM_F32 ? (const void*)((const float*)A.t.qkv + t * A.t.qkv_stride) : (const void*)((const uint16_t*)A.t.qkv + t * A.t.qkv_stride);
}
/* Values i..i+3 and i+D/2..i+D/2+3 of head h of a row, turned by the angles of position pos where `turn`. */
template <int SRC, int D>
__device__ __forceinline__ void app_pair(const app_args& A, const void* row, int h, int i, bool turn, int64_t pos, float (&a)[4], float (&b)[4]) {
    app_load4<SRC>(row, (int64_t)h * D + i, a);
    app_load4<SRC>(row, (int64_t)h * D + i + D / 2, b);
    if (turn) {
        const bl_v4f c = *bl_gc<bl_v4f>(A.t.cos + pos * (D / 2) + i), s = *bl_gc<bl_v4f>(A.t.sin + pos * (D / 2) + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = a[j], y = b[j];
            a[j] = x * c[j] - y * s[j];
            b[j] = y * c[j] + x * s[j];
        }
    }
}

/* A value as its code (the low 8 bits). */
template <int KIND>
__device__ __forceinline__ uint32_t app_code(float y) {
    constexpr float T = KIND == BL_KV_INT8 ? 127.0f : 448.0f;
    y = fminf(fmaxf(y, -T), T);                       /* (a NaN becomes -T) */
    if (KIND == BL_KV_INT8) return (uint32_t)(int)rintf(y) & 0xff;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xff;
}
template <int KIND>
__device__ __forceinline__ float app_value(uint32_t c) {
    return KIND == BL_KV_INT8 ? (float)(int8_t)c : __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
}
template <int KIND>
__device__ __forceinline__ uint32_t app_word(const float (&y)[4], float inv) {
    return app_code<KIND>(y[0] * inv) | app_code<KIND>(y[1] * inv) << 8 | app_code<KIND>(y[2] * inv) << 16 | app_code<KIND>(y[3] * inv) << 24;
}
/* The first `bytes` (1..4) codes of a word moved to a scale that is 1/ratio times as large; the other bytes are not written. */
template <int KIND>
__device__ __forceinline__ void app_move(uint8_t* p, int bytes, float ratio) {
    if (bytes == 4) {
        const uint32_t w = *(const uint32_t*)p;
        uint32_t o = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) o |= app_code<KIND>(app_value<KIND>((w >> (8 * j)) & 0xff) * ratio) << (8 * j);
        *(uint32_t*)p = o;
    } else {
        for (int j = 0; j < bytes; ++j) p[j] = (uint8_t)app_code<KIND>(app_value<KIND>(p[j]) * ratio);
    }
}

/* K and V: a run is the rows that go to one block (row t + k to the slot k further).  A workgroup looks at `window` rows, one a
 * lane, and does the runs that start there, WAVES waves for K or V of a head, 4 / WAVES of these beside each other: a unit's values
 * (block x D fp32 at most) stay in registers between the maximum and the rounding, so that a row is read once.
 * A thread has four values of a row and their rotary partners, D / 8 threads a row, NP rows.
 * Bound by HBM for prompts: 4096 tokens of 20 + 5 heads of 128 from fp32, 91 MB, 20.7 us = 4.4 TB/s (a large copy: 4.7); 19613 tokens of
 * 32 + 8 heads of 64 from bf16 into blocks of 16, 226 MB, 60 us = 3.8.  By the launch and the chain slots -> rows -> maximum -> codes for single tokens: 4.2 us. */
template <int SRC, int KIND, int D, int NP, int WAVES>
__device__ __forceinline__ void app_cache_rows(const app_args& A, int64_t first, int pair) {
    constexpr int UNITS = APP_THREADS / BL_WAVE / WAVES;
    constexpr int TPR = D / 8, UT = WAVES * BL_WAVE, ROWS = UT / TPR;   /* threads a row, threads a unit, rows a pass */
    constexpr float T = KIND == BL_KV_INT8 ? 127.0f : 448.0f;
    constexpr int PITCH = NP * ROWS + 4;                                /* of a feature's codes in LDS: 4 bytes more, other banks */
    __shared__ float s_max[APP_THREADS / BL_WAVE];
    __shared__ uint32_t s_v[UNITS][D * PITCH / 4];
    const bl_kv_cache& C = A.t.cache;
    const int lane = threadIdx.x & 63, H = C.n_kv, bs = 1 << A.shift;
    const int unit = (int)threadIdx.x / UT, tid = (int)threadIdx.x % UT;
    const int which = pair * UNITS + unit;                              /* kv head * 2 + (0: K, 1: V) */
    const bool live = which < 2 * H, is_v = which & 1;
    const int h = live ? which >> 1 : 0, head = A.t.n_q + (is_v ? H : 0) + h;
    const int sub = tid % TPR, rowi = tid / TPR, i4 = sub * 4;
    const int64_t T_all = A.t.T;
    /* Slots and positions of the rows around, all that this needs of them, in one go: [0..2] are the rows from `first` on,
     * [3..4] those in front of it, downwards.  What goes nowhere has the slot -1. */
    constexpr int SETS = 5;
    int slots[SETS], places[SETS];
    {
        int64_t at[SETS];
        bool in[SETS];
#pragma unroll
        for (int k = 0; k < SETS; ++k) {
            at[k] = k < 3 ? first + 64 * k + lane : first - 1 - 64 * (k - 3) - lane;
            in[k] = at[k] >= 0 && at[k] < T_all && (bs == 128 || (k != 2 && k != 4));      /* (a block of 64 ends within 80 rows) */
            slots[k] = in[k] ? A.t.slots[at[k]] : -1;
            places[k] = in[k] && A.t.cos ? A.t.positions[at[k]] : 0;
        }
        if (A.t.bad && pair == 0 && threadIdx.x < A.window && in[0] &&
            (slots[0] < -1 || (int64_t)slots[0] >= C.n_blocks << A.shift || (A.t.cos && (places[0] < 0 || places[0] >= A.t.n_pos))))
            atomicAdd(A.t.bad, 1);
#pragma unroll
        for (int k = 0; k < SETS; ++k)
            if (slots[k] < 0 || (int64_t)slots[k] >= C.n_blocks << A.shift || (A.t.cos && (places[k] < 0 || places[k] >= A.t.n_pos))) slots[k] = -1;
    }
    uint64_t todo = __ballot(lane < A.window && slots[0] >= 0);
    while (todo) {
        const int l0 = __builtin_ctzll(todo);
        const int64_t t0 = first + l0;
        const int slot = __builtin_amdgcn_readlane(slots[0], l0), off = slot & (bs - 1);
        /* The block's rows, a bit each: row t0 + k goes to the slot k further (one may be missing: a slot of -1, a bad position).
         * The first of them does the block. */
        uint64_t m0, m1;
        {
            auto member = [&](int set, int k) { return slots[set] >= 0 && slots[set] == slot + k && off + k >= 0 && off + k < bs; };
            const uint64_t a0 = __ballot(member(0, lane - l0)), a1 = __ballot(member(1, 64 + lane - l0)), a2 = bs == 128 ? __ballot(member(2, 128 + lane - l0)) : 0;
            m0 = l0 ? a0 >> l0 | a1 << (64 - l0) : a0;
            m1 = l0 ? a1 >> l0 | a2 << (64 - l0) : a1;
            todo &= ~a0;                                                /* (none of these begins another run) */
            uint64_t earlier = __ballot(member(3, -1 - lane - l0));
            if (bs == 128) earlier |= __ballot(member(4, -65 - lane - l0));
            if (earlier) continue;
        }
        const int n = m1 ? 128 - __builtin_clzll(m1) : 64 - __builtin_clzll(m0);
        auto has = [&](int r) { return r < n && (((r < 64 ? m0 : m1) >> (r & 63)) & 1); };
        const int64_t blk = slot >> A.shift;
        float* where = (is_v ? C.v_scale : C.k_scale) + blk * C.scale_stride + h;
        uint8_t* codes = (uint8_t*)(is_v ? C.v : C.k) + blk * (is_v ? C.v_stride : C.k_stride) + ((int64_t)h << A.shift) * D;
        /* values and their maximum */
        const float old = off > 0 ? *where : 0.0f;
        float a[NP][4], b[NP][4], most = 0.0f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int r = p * ROWS + rowi;
            int place = 0;                                              /* the row's position, from the lane that has it */
            if (A.t.cos) {
                place = __shfl(places[0], (l0 + r) & 63);
                const int next = __shfl(places[1], (l0 + r) & 63);
                if (l0 + r >= 64) place = next;
                if (bs == 128) {
                    const int third = __shfl(places[2], (l0 + r) & 63);
                    if (l0 + r >= 128) place = third;
                }
            }
            if (live && has(r)) app_pair<SRC, D>(A, app_row<SRC>(A, t0 + r), head, i4, !is_v && A.t.cos, place, a[p], b[p]);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) a[p][j] = b[p][j] = 0.0f;
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(fabsf(a[p][j]), fabsf(b[p][j])));   /* fmaxf passes over a NaN */
        most = bl_wave_max(most);
        if (WAVES > 1) {
            __syncthreads();                                            /* (s_max and s_v of the run before are read) */
            if (lane == 0) s_max[threadIdx.x >> 6] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, s_max[unit * WAVES + w]);
        }
        float scale = fmaxf(most, 1e-5f) * (1.0f / T);
        if (off > 0) {
            if (scale > old) {
                /* what the block holds moves to the larger scale */
                const float ratio = bl_div_rn(old, scale);
                if (live && !is_v) {
                    for (int i = tid; i < off * D / 4; i += UT) app_move<KIND>(codes + 4 * i, 4, ratio);
                } else if (live) {
                    const int words = (off + 3) / 4;
                    for (int i = tid; i < D * words; i += UT) {
                        const int d = i / words, w = i % words, left = off - 4 * w;
                        app_move<KIND>(codes + ((int64_t)d << A.shift) + 4 * w, left < 4 ? left : 4, ratio);
                    }
                }
            } else {
                scale = fmaxf(scale, old);
            }
        }
        if (live && tid == 0) *where = scale;                           /* (every thread of the unit has read the old one in front of the maximum) */
        const float inv = bl_div_rn(1.0f, scale);
        if (!is_v) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int r = p * ROWS + rowi;
                if (live && has(r)) {
                    uint8_t* o = codes + (off + r) * D + i4;
                    *(uint32_t*)o = app_word<KIND>(a[p], inv);
                    *(uint32_t*)(o + D / 2) = app_word<KIND>(b[p], inv);
                }
            }
        } else if (n == 1) {
            if (live && rowi == 0) {
                const uint32_t lo = app_word<KIND>(a[0], inv), hi = app_word<KIND>(b[0], inv);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    codes[((int64_t)(i4 + j) << A.shift) + off] = (uint8_t)(lo >> (8 * j));
                    codes[((int64_t)(i4 + D / 2 + j) << A.shift) + off] = (uint8_t)(hi >> (8 * j));
                }
            }
        } else {
            /* through LDS, where a feature's codes come to stand together as they do in the block (token offset as byte) */
            uint8_t* sv = (uint8_t*)s_v[unit];
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int r = p * ROWS + rowi;
                if (has(r)) {
                    const uint32_t lo = app_word<KIND>(a[p], inv), hi = app_word<KIND>(b[p], inv);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sv[(i4 + j) * PITCH + off + r] = (uint8_t)(lo >> (8 * j));
                        sv[(i4 + D / 2 + j) * PITCH + off + r] = (uint8_t)(hi >> (8 * j));
                    }
                }
            }
        }
        if (n > 1) {
            __syncthreads();
            if (live && is_v) {
                const uint8_t* sv = (const uint8_t*)s_v[unit];
                const int lw = A.shift - 2, words = 1 << lw, w0 = off / 4, w1 = (off + n + 3) / 4;
                for (int i = tid; i < D << lw; i += UT) {
                    const int d = i >> lw, w = i & (words - 1);
                    if (w < w0 || w >= w1) continue;
                    const uint8_t* from = sv + d * PITCH + 4 * w;
                    uint8_t* to = codes + 4 * i;
                    const int r = 4 * w - off;
                    if (r >= 0 && has(r) && has(r + 1) && has(r + 2) && has(r + 3)) {
                        *(uint32_t*)to = *(const uint32_t*)from;
                    } else {
                        for (int j = 0; j < 4; ++j)
                            if (r + j >= 0 && has(r + j)) to[j] = from[j];
                    }
                }
            }
            if (WAVES == 1) __syncthreads();                            /* s_v is free again */
        }
    }
}

/* Eight consecutive values of a row. */
template <int SRC>
__device__ __forceinline__ void app_load8(const void* row, int64_t i, float (&v)[8]) {
    if (SRC == BL_KV_FROM_F32) {
        float a[4], b[4];
        app_load4<SRC>(row, i, a), app_load4<SRC>(row, i + 4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
    } else {
        const app_v4u x = *bl_gc<app_v4u>((const uint16_t*)row + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[2 * j] = bl_bf16_to_f32(x[j] & 0xffff), v[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
    }
}
/* Q: a thread has eight values and their partners, the same ones of APP_HEADS heads of a row (their angles are read once). */
#define APP_HEADS 2
template <int SRC, int D>
__device__ __forceinline__ void app_query_units(const app_args& A, uint32_t u, uint32_t units_row, uint32_t all) {
    constexpr int TPH = D / 16;                                         /* threads a head */
    if (u >= all) return;
    const uint32_t t = u / units_row, r = u % units_row;
    const int h0 = (int)(r / TPH) * APP_HEADS, i = (int)(r % TPH) * 8;
    const int64_t pos = A.t.cos ? A.t.positions[t] : 0;
    const bool there = !A.t.cos || (pos >= 0 && pos < A.t.n_pos);
    const void* row = app_row<SRC>(A, t);
    float a[APP_HEADS][8], b[APP_HEADS][8], c[8], s[8];
#pragma unroll
    for (int k = 0; k < APP_HEADS; ++k)
        if (h0 + k < A.t.n_q) {
            app_load8<SRC>(row, (int64_t)(h0 + k) * D + i, a[k]);
            app_load8<SRC>(row, (int64_t)(h0 + k) * D + i + D / 2, b[k]);
        }
    if (A.t.cos && there) {
        app_load8<BL_KV_FROM_F32>(A.t.cos + pos * (D / 2), i, c);
        app_load8<BL_KV_FROM_F32>(A.t.sin + pos * (D / 2), i, s);
    }
#pragma unroll
    for (int k = 0; k < APP_HEADS; ++k)
        if (h0 + k < A.t.n_q) {
            if (A.t.cos) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = a[k][j], y = b[k][j];
                    a[k][j] = there ? x * c[j] - y * s[j] : 0.0f;
                    b[k][j] = there ? y * c[j] + x * s[j] : 0.0f;
                }
            }
            uint16_t* o = A.t.q_out + (int64_t)t * A.t.q_stride + (h0 + k) * D + i;
            *bl_g((app_v4u*)o) = (app_v4u){bl_pack2_bf16(a[k][0], a[k][1]), bl_pack2_bf16(a[k][2], a[k][3]), bl_pack2_bf16(a[k][4], a[k][5]), bl_pack2_bf16(a[k][6], a[k][7])};
            *bl_g((app_v4u*)(o + D / 2)) = (app_v4u){bl_pack2_bf16(b[k][0], b[k][1]), bl_pack2_bf16(b[k][2], b[k][3]), bl_pack2_bf16(b[k][4], b[k][5]), bl_pack2_bf16(b[k][6], b[k][7])};
        }
}

/* Workgroups of K and V (window x head pairs) first, those of Q behind them. */
template <int SRC, int KIND, int D, int NP, int WAVES>
__global__ __launch_bounds__(APP_THREADS) void bl_kv_append_kernel(app_args A, int kv_blocks, uint32_t units_row, uint32_t all) {
    const int x = (int)blockIdx.x;
    if (x < kv_blocks) {
        /* Consecutive workgroups go to the eight dies in turn, and the windows in which runs start are evenly spaced: each die takes
         * a contiguous eighth of the windows, else a few dies have all the work (4096 tokens 37 -> 22 us). */
        const int pairs = kv_blocks / A.windows, die = x & 7, part = kv_blocks >> 3, more = kv_blocks & 7;
        const int at = die * part + (die < more ? die : more) + (x >> 3);
        app_cache_rows<SRC, KIND, D, NP, WAVES>(A, (int64_t)(at / pairs) * A.window, at % pairs);
    }
    else app_query_units<SRC, D>(A, (uint32_t)(x - kv_blocks) * APP_THREADS + threadIdx.x, units_row, all);
}

template <int SRC, int KIND, int D, int NP, int WAVES>
static bl_status app_launch(const app_args& A, hipStream_t st) {
    constexpr int UNITS = APP_THREADS / BL_WAVE / WAVES;
    const int64_t units_row = A.t.q_out ? (int64_t)((A.t.n_q + APP_HEADS - 1) / APP_HEADS) * (D / 16) : 0, all = A.t.T * units_row;
    const int64_t kv = (int64_t)A.windows * ((2 * A.t.cache.n_kv + UNITS - 1) / UNITS), q = (all + APP_THREADS - 1) / APP_THREADS;
    if (all > 0xf0000000ll || kv + q > 0x7fffffff) return BL_ERR_SHAPE;
    bl_kv_append_kernel<SRC, KIND, D, NP, WAVES><<<(unsigned)(kv + q), APP_THREADS, 0, st>>>(A, (int)kv, units_row ? (uint32_t)units_row : 1, (uint32_t)all);
    return BL_OK;
}
/* Waves and passes by the block's size: 1024 to 2048 values of a block and head are one wave's, 16384 four waves' in eight passes. */
template <int SRC, int KIND>
static bl_status app_choose(const app_args& A, hipStream_t st) {
    if (A.t.cache.head_dim == 128)
        return A.shift == 4 ? app_launch<SRC, KIND, 128, 4, 1>(A, st) : A.shift == 5 ? app_launch<SRC, KIND, 128, 4, 2>(A, st)
             : A.shift == 6 ? app_launch<SRC, KIND, 128, 4, 4>(A, st) : app_launch<SRC, KIND, 128, 8, 4>(A, st);
    return A.shift == 4 ? app_launch<SRC, KIND, 64, 2, 1>(A, st) : A.shift == 5 ? app_launch<SRC, KIND, 64, 4, 1>(A, st)
         : A.shift == 6 ? app_launch<SRC, KIND, 64, 4, 2>(A, st) : app_launch<SRC, KIND, 64, 4, 4>(A, st);
}

extern "C" bl_status bl_kv_append(const bl_kv_tokens* t, bl_stream s) {
    if (!t || !t->qkv || !t->slots) return BL_ERR_NULL;
    if (const bl_status rc = bl_kv_cache_check(&t->cache)) return rc;
    if (!t->cos != !t->sin || (t->cos && !t->positions)) return BL_ERR_NULL;
    if (t->qkv_kind != BL_KV_FROM_F32 && t->qkv_kind != BL_KV_FROM_BF16) return BL_ERR_VALUE;
    const int D = t->cache.head_dim, unit = t->qkv_kind == BL_KV_FROM_F32 ? 4 : 8;
    const int64_t most = (int64_t)1 << 40;
    if (t->T < 1 || t->T > BL_MAX_DIM || t->n_q < 0 || t->n_q > 65535 || t->qkv_stride < (t->n_q + 2 * (int64_t)t->cache.n_kv) * D || t->qkv_stride > most ||
        (t->cos && (t->n_pos < 1 || t->n_pos > 0x7fffffff)) || (t->q_out && (t->n_q < 1 || t->q_stride < (int64_t)t->n_q * D || t->q_stride > most)))
        return BL_ERR_SHAPE;
    if (!bl_aligned(t->qkv, 16) || t->qkv_stride % unit || !bl_aligned(t->cos, 16) || !bl_aligned(t->sin, 16) || !bl_aligned(t->slots, 4) ||
        !bl_aligned(t->positions, 4) || !bl_aligned(t->bad, 4) || !bl_aligned(t->q_out, 16) || (t->q_out && t->q_stride % 8))
        return BL_ERR_ALIGN;
    app_args A = {*t, bl_log2(t->cache.block), 1, 0};
    /* rows a K/V workgroup: one where they are few (each is a run of its own in a decode step), more where they are many (the
     * runs of prompts start in few windows, and a workgroup without one is not free).  Windows of 1, 2, 4, 8 and 16 rows, us: 64 single tokens 5.0, 6.2,
     * 9.4, 16, 29; 1024 of them 25, 22, 23, 24, 37; 4096 104, 88, 80, 79, 90; a prompt of 512 13, 8.4, 8.4, 8.3, 8.3; of 1024 25, 15, 11.4, 10.3, 10.1;
     * of 4096 92, 55, 36, 26, 21. */
    while (A.window < 16 && t->T > 256 * A.window) A.window *= 2;
    A.windows = (int)((t->T + A.window - 1) / A.window);
    const hipStream_t st = (hipStream_t)s;
    const bool f32 = t->qkv_kind == BL_KV_FROM_F32, i8 = t->cache.kind == BL_KV_INT8;
    const bl_status rc = f32 ? i8 ? app_choose<BL_KV_FROM_F32, BL_KV_INT8>(A, st) : app_choose<BL_KV_FROM_F32, BL_KV_E4M3>(A, st)
                             : i8 ? app_choose<BL_KV_FROM_BF16, BL_KV_INT8>(A, st) : app_choose<BL_KV_FROM_BF16, BL_KV_E4M3>(A, st);
    if (rc) return rc;
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}
