// What the library was built from.  A file of its own: the digest changes with every source, and nothing else needs compiling for that.
#include "../../include/cusa.h"

#ifndef CUSA_BUILD_ID
#define CUSA_BUILD_ID "unknown"
#endif
// The marker also lets a loader read the id from the file without mapping the library.
static const char kBuildId[] = "CUSA_BUILD_ID=" CUSA_BUILD_ID;
extern "C" const char* cusa_build_id(void) { return kBuildId + 14; }
