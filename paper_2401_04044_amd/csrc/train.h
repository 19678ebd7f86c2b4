// Internal: scratch sizes of the training calls (train.hip).
#pragma once
#include "../../include/ffsplit.h"
#include <stddef.h>
#include <stdint.h>

namespace ffsplit {
size_t train_workspace_bytes(const ffsplit_desc_t* d, int32_t call_id, int64_t T);
}  // namespace ffsplit
