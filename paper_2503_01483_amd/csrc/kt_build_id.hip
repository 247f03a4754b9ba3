// kt_build_id.hip -- the id of the sources, in a file of its own: a build script may keep the other objects.
#include "../../include/kt.h"

#ifndef KT_BUILD_ID
#define KT_BUILD_ID "unknown"
#endif

extern "C" const char* kt_build_id(void) { return KT_BUILD_ID; }
