// Attention for a tree of drafted tokens: its entry points refuse every call until the kernel is there.
#include "../../include/pdattn.h"
extern "C" {
pdattn_status pdattn_tree_workspace_size(int, int, int, int, int, size_t*) { return PDATTN_UNSUPPORTED; }
pdattn_status pdattn_decode_tree(const pdattn_args*, const int32_t*, int, const uint64_t*, int, pdattn_stream_t) { return PDATTN_UNSUPPORTED; }
pdattn_status pdattn_decode_tree_fp8(const pdattn_args*, const int32_t*, int, const uint64_t*, int, const float*, const float*, pdattn_stream_t) { return PDATTN_UNSUPPORTED; }
}
