// gba_window_attention.hip -- attention of each request's new tokens over a
// paged cache: the kernels with a window and sinks.
#include "gba_tree_kernel.hpp"

using namespace gba;

extern "C" gba_status gba_window_attention_workspace_size(const gba_attention *desc, int64_t window, int64_t sinks, size_t *bytes)
{
    return attend_workspace_size<true>(desc, window, sinks, bytes);
}

extern "C" gba_status gba_window_attention(const gba_attention *desc, int64_t window, int64_t sinks, gba_stream_t stream)
{
    return attend<true>(desc, window, sinks, stream);
}
