// The streaming projection of a few rows (decode_bf16.hip), for calls that are not a draft step on a contiguous cache.  Not part of
// the public interface.
#pragma once
#include "common.h"

namespace beagle {

constexpr int PROJ_ROWS = 64;              // rows of a streaming projection, at most
// y = x W for up to PROJ_ROWS rows (kv_append_bf16_fits), split over k; ws: half of kv_append_bf16_ws_bytes
void launch_proj_rows_bf16(const void* x, const void* w, void* y, int32_t n, int32_t N, int32_t K, void* ws, const char* name, hipStream_t s);
// The same with the rows of each head (128 wide) rotated: the finished float sums are, so a value rounds once.  rope.pos: of every row;
// rope.tab: room for n rows
void launch_proj_rope_rows_bf16(const void* x, const void* w, void* y, int32_t n, int32_t N, int32_t K, void* ws, const RopeRows& rope,
                                const char* name, hipStream_t s);

}  // namespace beagle
