// Shared by the entry points of the paged MXFP4 cache (private; the public ABI is include/mx4.h).
#pragma once

#include "mx_common.h"
#include "mx_kv_layout.h"

namespace mx {

constexpr int64_t kKvMost = (int64_t)1 << 30;       // tokens of a call
constexpr int64_t kKvMostHeads = (int64_t)1 << 16;
constexpr int64_t kKvMostWaves = ((int64_t)1 << 26) - 4;  // of a launch in workgroups of four: fewer than 2^32 work-items, the last workgroup whole

inline bool kv_head_dim(int64_t D) { return D == 64 || D == 96 || D == 128 || D == 192 || D == 256; }

// The arrays of a cache.  k_mbs and v_mbs are both there or both not.
struct KvArrays {
    uint8_t *k_codes, *k_scales, *k_mbs, *v_codes, *v_scales, *v_mbs;
    KvLayout at;
    int check(int64_t num_pages, int64_t page_size, int64_t Hkv, int64_t D) const;
    void shape(int64_t page_size, int64_t Hkv, int64_t D);
};

}  // namespace mx
