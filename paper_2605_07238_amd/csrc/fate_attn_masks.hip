// The row tile kernel with documents, windows and prefixes: its own file, so that
// the instances compile side by side.
#define FATE_ATTN_SHAPE 1
#include "fate_attn_tile.hip"
