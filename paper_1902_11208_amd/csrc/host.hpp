// Shared by the files of the host layer.
#pragma once

#include <stddef.h>

#include "mdlstm.h"

namespace mdl {

// Keeps `message` for mdlstm_last_error() on this thread and returns `st`.
mdlstm_status set_error(mdlstm_status st, const char* message);

// The debug mode MDLSTM_POISON_WORKSPACE=1: fills a workspace of floating-point
// numbers with NaN; otherwise nothing.
mdlstm_status poison_workspace(void* ws, size_t bytes, void* stream);

}  // namespace mdl
