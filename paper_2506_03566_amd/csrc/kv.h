// Paged caches of a program's own (poss_kv_cache): how kernels see them, and what every call checks (rotary.hip, kv_attend.hip, kv_evict.hip).
#pragma once
#include "../../include/poss.h"
#include "device_utils.h"

namespace poss {

int set_error(int code, const char *fmt, ...);     // notes the message for poss_last_error(NULL), returns code

struct KvView {
    void *k, *v;
    const int32_t *table;
    int64_t k_page, v_page;              // values from a page to the next
    int table_stride, slots;             // slots of a sequence
    int n_pages, n_seq, hkv, dh, shift;  // shift: log2 of a page's tokens
};

static inline KvView kv_view(const poss_kv_cache &c) {
    const int shift = c.page_tokens == 32 ? 5 : c.page_tokens == 64 ? 6 : 7;
    return KvView{c.k, c.v, c.page_table, c.k_page_stride, c.v_page_stride, c.table_stride, c.table_pages << shift, c.n_pages, c.n_seq, c.n_kv_heads, c.head_dim, shift};
}

// The page of a sequence's slot, -1 where there is none.
__device__ __forceinline__ int kv_page(const KvView &c, int b, int slot) {
    if ((unsigned)slot >= (unsigned)c.slots) return -1;
    const int pg = c.table[(int64_t)b * c.table_stride + (slot >> c.shift)];
    return (unsigned)pg < (unsigned)c.n_pages ? pg : -1;
}
// Element offsets of a slot's key, and of row d of the transposed values at a slot (page valid).
__device__ __forceinline__ int64_t kv_key_at(const KvView &c, int page, int head, int slot) {
    return page * c.k_page + ((int64_t)(head << c.shift) + (slot & ((1 << c.shift) - 1))) * c.dh;
}
__device__ __forceinline__ int64_t kv_value_at(const KvView &c, int page, int head, int d, int slot) {
    return page * c.v_page + ((int64_t)(head * c.dh + d) << c.shift) + (slot & ((1 << c.shift) - 1));
}

static inline bool kv_aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
static inline bool kv_bad_dtype(int32_t t) { return t < 0 || t > 2; }

static inline int kv_launched(const char *who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? POSS_OK : set_error(POSS_E_HIP, "%s: %s", who, hipGetErrorString(e));
}

// Why the kernels do not take this cache (nullptr: they do).  Pointers are looked at only where there are sequences.
static inline const char *kv_cache_bad(const poss_kv_cache *c) {
    if (!c) return "no cache";
    if (kv_bad_dtype(c->dtype)) return "bad type";
    if (c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->head_dim < 32 || c->head_dim > 256 || c->head_dim % 32) return "head_dim must be a multiple of 32 up to 256, heads 1 to 65535";
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return "page_tokens must be 32, 64 or 128";
    if (c->n_pages < 1 || c->n_seq < 0 || c->n_seq > 65535 || c->table_pages < 1 || (int64_t)c->table_pages * c->page_tokens > 1 << 30 || c->table_stride < c->table_pages)
        return "bad pages or sequences";
    const int64_t page = (int64_t)c->n_kv_heads * c->page_tokens * c->head_dim, whole = 16 / (int64_t)dtype_size(c->dtype);
    if (c->n_pages > 1 && (c->k_page_stride < page || c->v_page_stride < page)) return "pages overlap";
    if (c->k_page_stride % whole || c->v_page_stride % whole) return "pages must lie whole 16 bytes apart";
    if (c->n_seq == 0) return nullptr;
    if (!c->k || !c->v || !c->page_table) return "null argument";
    if (!kv_aligned(c->k, 16) || !kv_aligned(c->v, 16) || !kv_aligned(c->page_table, 4)) return "keys and values must be aligned to 16 bytes, the page table to 4";
    return nullptr;
}

}  // namespace poss
