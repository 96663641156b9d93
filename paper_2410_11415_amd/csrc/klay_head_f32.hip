// The head of a network in f32.
#include "klay_head_launch.hip.h"

KLAY_HEAD(f32)
