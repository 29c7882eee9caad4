// The row tile kernel with shaped scores: its own file so that the two halves
// of the instances compile side by side.
#define FATE_ATTN_SHAPED 1
#include "fate_attn_tile.hip"
