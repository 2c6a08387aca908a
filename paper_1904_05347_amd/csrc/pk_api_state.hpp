// pk_api_state.hpp -- the calling thread's "last" answers (pk_api.hip holds
// them), for the C entry points in other files.
#pragma once

namespace pk {

void api_begin();                  // no invalid argument, no configuration yet
int api_invalid(int position);     // PK_ERR_INVALID_VALUE at this 1-based position
void api_ran(const char *config);  // the configuration the call ran (static storage)

}  // namespace pk
