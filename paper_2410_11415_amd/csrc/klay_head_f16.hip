// The head of a network in f16.
#include "klay_head_launch.hip.h"

KLAY_HEAD(f16)
