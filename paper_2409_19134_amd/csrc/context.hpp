// What the library's parts share of a context.
#pragma once
#include "../../include/spd.h"

namespace spd {

struct TokensState;  // tables and scratch memory of the calls for several tokens per user (tokens_api.hip)

struct ContextBase {
    int device = 0;
    int n_cus = 0;
    int last_hip = 0;
    int cache_entries = 0;                         // views remembered per entry point
    TokensState *tokens = nullptr;                 // made by the first such call
    void (*tokens_free)(TokensState *) = nullptr;  // set with it
};

// The context behind a handle, for the parts that do not know the rest of it.
__attribute__((visibility("hidden"))) ContextBase *context_base(spd_ctx *ctx);

}  // namespace spd
