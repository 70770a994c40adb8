// Routing of tokens to experts whose logits are of type BAGUA_F32.
#include "route_device.hpp"

namespace bagua {

template int launch_route<BAGUA_F32>(Lists<kRouteLists>&, RouteArgs, const size_t*, int, hipStream_t);
template int launch_route_grad<BAGUA_F32>(Lists<kRouteGradLists>&, RouteGradArgs, const size_t*, int, hipStream_t);

}  // namespace bagua
