// The status of a HIP call's result; a failed call's code is kept for ecspmv_last_hip_error.
#ifndef ECSPMV_STATUS_H
#define ECSPMV_STATUS_H

namespace ecs {
int hip_status(int hip_error);
}
#endif
