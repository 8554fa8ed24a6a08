// What the paged cache's operators share on the host side.
#pragma once

namespace specsteer {

// SM count of the current device (read once per device); 0 on failure.
int current_sm_count();

}  // namespace specsteer
