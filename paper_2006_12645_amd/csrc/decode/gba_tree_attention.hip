// gba_tree_attention.hip -- attention of each request's new tokens over a paged
// cache: the kernels without a window.
#include "gba_tree_kernel.hpp"

using namespace gba;

extern "C" gba_status gba_tree_attention_workspace_size(const gba_attention *desc, size_t *bytes)
{
    return attend_workspace_size<false>(desc, 0, 0, bytes);
}

extern "C" gba_status gba_tree_attention(const gba_attention *desc, gba_stream_t stream)
{
    return attend<false>(desc, 0, 0, stream);
}
