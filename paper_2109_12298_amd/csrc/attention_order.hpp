// The order of blocks whose work differs by documents: see attention_order.hip.
#pragma once

#include "attention.hpp"

namespace dpg {
namespace attn {

// Whether blocks of 128 rows (keys) are worth an order, and its entries (0: none).
i64 row_order_entries(const dp_attention &a);
i64 key_order_entries(const dp_attention &a);
// rows, keys: orders to write, or NULL
void order_blocks(const Call &c, int32_t *rows, int32_t *keys, hipStream_t stream);

}  // namespace attn
}  // namespace dpg
