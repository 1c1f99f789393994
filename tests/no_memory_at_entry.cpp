// Calls whose host memory has run out where they report what they refuse: they return, and no exception leaves them.  No GPU: refused calls
// launch nothing.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>

#include "../include/fuse.h"

static bool none = false;

void *operator new(std::size_t n)
{
    void *p = none ? nullptr : std::malloc(n);
    if (!p)
        throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }

static int bad = 0;
#define EXPECT(call, want)                                                                         \
    do {                                                                                           \
        none = true;                                                                               \
        const long long got = (long long)(call);                                                   \
        none = false;                                                                              \
        if (got != (long long)(want) || std::strcmp(fuse_last_error(), "out of memory")) {         \
            std::printf("%s: %lld, \"%s\"\n", #call, got, fuse_last_error());                      \
            bad = 1;                                                                               \
        }                                                                                          \
    } while (0)

int main()
{
    fuse_attn attn = {};
    fuse_block block = {};
    fuse_rotary rotary = {};
    fuse_cache cache = {};
    fuse_cache_query query = {};
    attn.dtype = block.dtype = rotary.dtype = cache.dtype = 99;            // refused, with a text that takes an allocation
    fuse_tensor tensor = {};
    tensor.count = -1;
    fuse_attention_bytes(&attn);                                           // (the thread's text, once)
    EXPECT(fuse_attention_bytes(&attn), 0);
    EXPECT(fuse_attention_backward_bytes(&attn), 0);
    EXPECT(fuse_attention_shaped_backward_bytes(&attn, nullptr), 0);
    EXPECT(fuse_qk_rotary_backward_bytes(&rotary), 0);
    EXPECT(fuse_attention_cache_bytes(&cache, &query), 0);
    EXPECT(fuse_attention(&attn, nullptr, 0, 0, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_attention_backward(&attn, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_attention_shaped(&attn, nullptr, nullptr, 0, 0, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_attention_shaped_backward(&attn, nullptr, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_attention_zero_rest(&attn, nullptr, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_qk_rotary(&rotary, nullptr, 0, 0, nullptr, 0, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_qk_rotary_backward(&rotary, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_cache_write(&cache, nullptr, 0, 0, nullptr, 0, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_attention_cache(&cache, &query, nullptr, 0, 0, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_block_norm(&block, nullptr, 0, nullptr, 0, nullptr, 0, nullptr), FUSE_ENOMEM);
    EXPECT(fuse_grad_norm(&tensor, 1, nullptr, nullptr, 0, nullptr), FUSE_ENOMEM);
    fuse_expr expr = {};
    fuse_dense x = {};
    EXPECT(fuse_cell(&expr, &x, nullptr, -1, 99, nullptr, nullptr), FUSE_ENOMEM);
    return bad;
}
