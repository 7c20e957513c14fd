// The paged, ragged cache's host object and what its source files share (layout: rlkv_paged.cu).
#pragma once

#include <vector>

#include "rlkv_host.cuh"

struct rlkv_paged {
    int layers, kv_heads, q_heads, head_dim, max_seqs, n_pages, table_stride, sink, window;
    int max_seq_len;              // most tokens a sequence may hold (the page table is laid out for a few more)
    int device, sm_count, stages, groups, item_tiles;
    int rows_comp, max_batch, max_items, max_grid;
    int out_bf16;
    int step_mode;                // rlkv_paged_step: 0 chooses, 1 one decode launch per layer, 2 one for the whole step
    bool step_in_one_launch;      // the shape allows one decode launch for a whole step
    long long step_slots;         // partial records the scratch holds when both copies are used as one
    int fp8;                      // K/V rows (pages and rings) are held as E4M3 codes
    std::vector<float> k_scale, v_scale;  // [layers*kv_heads]
    std::vector<long long> page0_8, ring0_8;  // first full-head page / first ring page of each layer in the 8-bit pool
    long long pages8;                      // pages of the 8-bit pool
    size_t off_pool8, off_scales;
    CUtensorMap map_k;  // the 8-bit pool as rows of 128 bytes, one page per box
    CUtensorMap map_codes;  // and the K or the V codes of a page per box
    long long pool_rows;
    std::vector<uint8_t> is_full;
    std::vector<int> slot_of_head, head_of_slot;  // [layers*kv_heads]
    std::vector<int> n_full, n_comp;
    std::vector<long long> full_row0, comp_row0;
    std::vector<int> len;         // [layers][max_seqs]
    std::vector<int> table;       // [max_seqs][table_stride], -1 = no page
    std::vector<int> free_pages;  // stack of physical pages
    std::vector<uint8_t> open;    // [max_seqs]
    size_t off_pool, off_tables, off_head_table, off_layer_desc, off_slopes, off_page_table, off_tickets, off_status, off_partials, total;
    uint8_t* dev_base;
    bool owns_buffer;
    float *chunk_records, *own_records;  // scratch of rlkv_paged_chunk_attention; the library's own, once it is taken (or null)
    size_t chunk_bytes;
    bool chunk_settled;           // false: the next call that attends chunks takes own_records first
    CUtensorMap tmap;
    uint64_t launches;
    const float* rotary;          // rlkv_paged_set_rotary: the caller's table of angles (device), null: none set
    int rotary_rows, rotary_dim, rotary_interleaved;
    const float *q_norm, *k_norm; // rlkv_paged_set_norms: the caller's weights (device), null: none set
    float norm_eps;
    float softcap;                // rlkv_paged_set_scores: 0 no cap
    bool biased;                  // and whether scores are lowered by distance (slopes at off_slopes)
    bool has_slopes;              // whether slopes have ever been written
};

namespace rlkv {

template <typename T>
inline T* dev_at(const rlkv_paged* p, size_t off) { return reinterpret_cast<T*>(p->dev_base + off); }

inline bool valid_layer(const rlkv_paged* p, int layer) { return p && layer >= 0 && layer < p->layers; }
inline bool valid_slot(const rlkv_paged* p, int slot) { return slot >= 0 && slot < p->max_seqs && p->open[slot]; }

// The request slots of a call: all open, no slot twice.
inline int check_slots(const rlkv_paged* p, const int* slots, int n)
{
    if (!slots || n < 1 || n > p->max_batch) return RLKV_EINVAL;
    std::vector<uint8_t> seen(p->max_seqs, 0);
    for (int i = 0; i < n; ++i) {
        if (!valid_slot(p, slots[i]) || seen[slots[i]]) return RLKV_EINVAL;
        seen[slots[i]] = 1;
    }
    return RLKV_OK;
}

inline int* len_of(rlkv_paged* p, int layer) { return p->len.data() + (size_t)layer * p->max_seqs; }
inline const int* len_of(const rlkv_paged* p, int layer) { return p->len.data() + (size_t)layer * p->max_seqs; }

}  // namespace rlkv
