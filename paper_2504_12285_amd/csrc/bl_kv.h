/* Internal helpers of the key/value cache calls (bl_kv.hip, bl_attn.hip): host checks of the cache descriptor. */
#pragma once
#include "bl_host.h"

static inline bool bl_kv_block_ok(int64_t block) { return block == 16 || block == 32 || block == 64 || block == 128; }
static inline int bl_log2(int v) { return 31 - __builtin_clz((unsigned)v); }

static inline bl_status bl_kv_cache_check(const bl_kv_cache* c) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return BL_ERR_NULL;
    if (c->kind != BL_KV_INT8 && c->kind != BL_KV_E4M3) return BL_ERR_VALUE;
    if (!bl_kv_block_ok(c->block) || (c->head_dim != 64 && c->head_dim != 128) || c->n_kv < 1 || c->n_kv > 65535 || c->n_blocks < 1 ||
        c->n_blocks > (((int64_t)1 << 31) - 1) / c->block)
        return BL_ERR_SHAPE;
    const int64_t bytes = (int64_t)c->n_kv * c->block * c->head_dim, most = ((int64_t)1 << 36) - 16;
    if (c->k_stride < bytes || c->v_stride < bytes || c->scale_stride < c->n_kv || c->k_stride > most || c->v_stride > most || c->scale_stride > most)
        return BL_ERR_SHAPE;
    if (!bl_aligned(c->k, 16) || !bl_aligned(c->v, 16) || c->k_stride % 16 || c->v_stride % 16 || !bl_aligned(c->k_scale, 4) || !bl_aligned(c->v_scale, 4))
        return BL_ERR_ALIGN;
    return BL_OK;
}
