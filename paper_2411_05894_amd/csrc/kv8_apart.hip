// Attention over an 8-bit KV cache whose sequences share prefixes in groups, each sequence by itself: the shared blocks are read through the table of the group's first
// sequence, by every one of them.  Where a sequence's rows fill their tiles that costs less than joining partial results, since the blocks stay in the dies' caches.
#include "kv8_launch.h"

hipError_t launch_kv8_apart(Kv8SharedArgs a, int fmt, int d, void *ws, hipStream_t s) { return launch_attention<KV8_APART>(a, fmt, d, ws, s); }
