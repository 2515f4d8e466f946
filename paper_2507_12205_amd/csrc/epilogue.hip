// The product kernels with an epilogue: the same source, with what kernels.hip has under ECS_EPILOGUE; a unit of its own, so that both
// are compiled at the same time.  Clock stamps are taken of the products alone.
#undef ECS_TRACE
#define ECS_EPILOGUE 1
#include "kernels.hip"
