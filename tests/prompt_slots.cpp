// For test_prompt_slots.py: asks rm_slots.h for every slot, head and sequence of a call.
#include <cstdint>

#include "rm_slots.h"

// Every sequence is asked for in every slot, whatever a search would find there.
// Returns how many answers leave the call's arrays.
extern "C" int64_t out_of_range(const int32_t* offsets, int32_t n_seqs, int32_t n_tokens,
                                int32_t max_tokens, int32_t window, int32_t group,
                                int32_t kv_heads)
{
    const rm::SlotShape s = {n_tokens, max_tokens, window, group, kv_heads};
    const int64_t slots = (int64_t)n_tokens * group / rm::kTileRows + n_seqs;
    int64_t bad = 0;
    for (int b = 0; b < n_seqs; ++b)
        for (int64_t slot = 0; slot < slots; ++slot)
            for (int head = 0; head < kv_heads; ++head) {
                const int32_t begin = offsets[b], end = offsets[b + 1];
                const rm::SlotTile t = rm::tile_of(s, head, slot, b, begin, end);
                if (t.what == rm::SlotTile::CLEAR)
                    bad += t.clear_from < t.clear_upto &&
                           (t.clear_from < 0 || t.clear_upto > n_tokens);
                if (t.what != rm::SlotTile::ATTEND) continue;
                const int64_t count = (int64_t)end - begin;
                // the first key of every step is a row of the sequence
                bad += begin < 0 || end > n_tokens || t.first_row < 0 ||
                       t.first_row > t.last_row || t.last_row >= count * group ||
                       t.first_step < 0 || t.first_step >= t.end_step ||
                       (int64_t)(t.end_step - 1) * rm::kStepKeys >= count;
            }
    return bad;
}

// Counts into taken[n_tokens][kv_heads * group] how often a call's workgroups attend
// for a pair, and into cleared[n_tokens] how often they clear a row, where the offsets
// do not decrease: a slot is that of the last sequence that begins there or before.
extern "C" void rows_taken(const int32_t* offsets, int32_t n_seqs, int32_t n_tokens,
                           int32_t max_tokens, int32_t window, int32_t group, int32_t kv_heads,
                           int32_t* taken, int32_t* cleared)
{
    const rm::SlotShape s = {n_tokens, max_tokens, window, group, kv_heads};
    const int64_t slots = (int64_t)n_tokens * group / rm::kTileRows + n_seqs;
    for (int64_t slot = 0; slot < slots; ++slot) {
        int b = -1;
        while (b + 1 < n_seqs && rm::first_slot(s, offsets[b + 1], b + 1) <= slot) ++b;
        if (b < 0) continue;
        for (int head = 0; head < kv_heads; ++head) {
            const rm::SlotTile t = rm::tile_of(s, head, slot, b, offsets[b], offsets[b + 1]);
            if (t.what == rm::SlotTile::CLEAR)
                for (int64_t r = t.clear_from; r < t.clear_upto; ++r) ++cleared[r];
            if (t.what == rm::SlotTile::ATTEND)
                for (int r = t.first_row; r <= t.last_row; ++r)
                    ++taken[(int64_t)(offsets[b] + r / group) * kv_heads * group + head * group +
                            r % group];
        }
    }
}
