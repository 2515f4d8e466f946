// Attention of the nodes of a tree: the same source, with what attention.hip has under ECS_TREE; a unit of its own, so that both are compiled
// at the same time.
#define ECS_TREE 1
#include "attention.hip"
