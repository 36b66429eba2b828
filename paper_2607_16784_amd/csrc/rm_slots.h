// rm_slots.h -- which rows a workgroup of the packed prompts' attention takes
// (prompt.hip).  Plain arithmetic on the offsets, which are a caller's device data, so
// that a check on the host can ask it for every case.  Not part of the C ABI.
#pragma once

#include <cstdint>

namespace rm {

constexpr int kTileRows = 128;       // (token, query head) pairs of a tile
constexpr int kStepKeys = 64;        // keys of a step

struct SlotShape {
    int32_t n_tokens, max_tokens, window;
    int32_t group, kv_heads;         // query heads of a kv head
};

// Tiles of the sequences lie in a row of slots, sequence b's from
// floor(first row * group / kTileRows) + b on: that leaves each enough, whatever the
// lengths, where the offsets do not decrease.
constexpr int32_t row_within(int32_t offset, int32_t n_tokens)
{
    return offset < 0 ? 0 : offset > n_tokens ? n_tokens : offset;
}
constexpr int64_t first_slot(const SlotShape& s, int32_t offset, int b)
{
    return (int64_t)row_within(offset, s.n_tokens) * s.group / kTileRows + b;
}

// What a workgroup does for head `head` of the kv heads in a slot that lies among those
// of sequence b, rows begin .. end-1.
struct SlotTile {
    enum { NOTHING, CLEAR, ATTEND } what;
    int64_t clear_from, clear_upto;  // CLEAR: rows of out
    // ATTEND: pairs of the tile, counted within the sequence, and steps of its keys
    int32_t first_row, last_row, first_step, end_step;
};

constexpr SlotTile tile_of(const SlotShape& s, int head, int64_t slot, int b, int32_t begin,
                           int32_t end)
{
    SlotTile t = {SlotTile::NOTHING, 0, 0, 0, 0, 0, 0};
    const int64_t count = (int64_t)end - begin, at_slot = slot - first_slot(s, begin, b);
    // Offsets that decrease: a search by the first slots may name a sequence that begins
    // behind the slot, and nothing below counts backwards.
    if (at_slot < 0) return t;
    if (begin < 0 || end > s.n_tokens || count < 0 || count > s.max_tokens) {
        // its rows in range, a part each slot and head
        const int64_t lo = row_within(begin, s.n_tokens);
        const int64_t rows = row_within(end, s.n_tokens) - lo;
        const int64_t pairs = (int64_t)s.kv_heads * s.group, part = at_slot * s.kv_heads + head;
        const int64_t from = part * kTileRows / pairs;
        const int64_t upto = ((part + 1) * kTileRows - 1) / pairs + 1;
        t.what = SlotTile::CLEAR;
        t.clear_from = lo + (from < rows ? from : rows);
        t.clear_upto = lo + (upto < rows ? upto : rows);
        return t;
    }
    // the last tiles take the longest, so they come first
    const int64_t rows = count * s.group;
    const int64_t tile = (rows + kTileRows - 1) / kTileRows - 1 - at_slot;
    if (tile < 0) return t;
    const int64_t last = (tile + 1) * kTileRows < rows ? (tile + 1) * kTileRows : rows;
    t.what = SlotTile::ATTEND;
    t.first_row = (int32_t)(tile * kTileRows);
    t.last_row = (int32_t)last - 1;
    const int32_t first_pos = t.first_row / s.group, last_pos = t.last_row / s.group;
    const int32_t seen = s.window > 0 ? first_pos - s.window + 1 : 0;
    t.first_step = seen > 0 ? seen / kStepKeys : 0;
    t.end_step = last_pos / kStepKeys + 1;
    return t;
}

}  // namespace rm
