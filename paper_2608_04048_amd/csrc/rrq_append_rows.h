// Which rows (token, head) of a group of tokens the append rotates, free of device code.
#pragma once

#include <stdint.h>

namespace rrq_detail {

// Of the group's n tokens from token0 on those that belong to sequences, which hold the
// batch's tokens first .. end - 1: rows begin .. end - 1 of the group, none where begin is
// not below end. Tokens are counted before they are multiplied by the heads: a group far
// from the sequences would pass 32 bits.
struct GroupRows {
    int32_t tokens, begin, end;
};
constexpr int32_t tokens_before(int64_t token0, int64_t at, int32_t n)
{
    return at <= token0 ? 0 : (at - token0 < n ? (int32_t)(at - token0) : n);
}
constexpr GroupRows group_rows(int64_t token0, int32_t n, int64_t first, int64_t end,
                               int32_t heads)
{
    return GroupRows{tokens_before(token0, end, n), tokens_before(token0, first, n) * heads,
                     tokens_before(token0, end, n) * heads};
}

}  // namespace rrq_detail
