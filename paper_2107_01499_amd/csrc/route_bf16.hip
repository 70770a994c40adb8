// Routing of tokens to experts whose logits are of type BAGUA_BF16.
#include "route_device.hpp"

namespace bagua {

template int launch_route<BAGUA_BF16>(Lists<kRouteLists>&, RouteArgs, const size_t*, int, hipStream_t);
template int launch_route_grad<BAGUA_BF16>(Lists<kRouteGradLists>&, RouteGradArgs, const size_t*, int, hipStream_t);

}  // namespace bagua
