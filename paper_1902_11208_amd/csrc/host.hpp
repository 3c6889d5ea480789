// Shared by the files of the host layer.
#pragma once

#include "mdlstm.h"

namespace mdl {

// Keeps `message` for mdlstm_last_error() on this thread and returns `st`.
mdlstm_status set_error(mdlstm_status st, const char* message);

}  // namespace mdl
