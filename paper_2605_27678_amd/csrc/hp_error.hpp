// Where a failing HIP call is noted for hp_last_hip_error, whichever file made it.
#pragma once

namespace hp {

void note_hip_error(int e);        // of this host thread

}  // namespace hp
