// The row tile kernel with capped and biased scores: its own file, so that the
// instances compile side by side.
#define FATE_ATTN_SHAPE 2
#include "fate_attn_tile.hip"
