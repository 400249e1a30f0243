// The bound workspace, for the calls outside ts_densify.hip that need one.  Hidden: no part of the C ABI.
#ifndef TS_WORKSPACE_H
#define TS_WORKSPACE_H

#include <stdint.h>

namespace ts_workspace {

// The bound workspace, to be written over in stream order; views of an earlier densify call into it are gone.
// TS_ERR_WORKSPACE if none is bound or it is smaller than bytes.
__attribute__((visibility("hidden"))) int take(int64_t bytes, void** ws);

}  // namespace ts_workspace

#endif  // TS_WORKSPACE_H
