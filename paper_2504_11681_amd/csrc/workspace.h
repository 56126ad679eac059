// The workspace that tfno_set_workspace registered last.
#pragma once
#include <stddef.h>

namespace tfno {

struct RegisteredWorkspace { void *ptr; size_t bytes; };
RegisteredWorkspace registered_workspace();

}  // namespace tfno
