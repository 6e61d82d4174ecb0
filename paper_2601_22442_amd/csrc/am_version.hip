// The library's version with the digest of its source files, in a file of its own: it is all that changes with every source.
#include "../../include/asyncmesh.h"

#ifndef AM_SOURCE_HASH
#define AM_SOURCE_HASH "unknown"
#endif

extern "C" const char *am_version(void) { return "asyncmesh-gfx950 0.2 src:" AM_SOURCE_HASH; }
