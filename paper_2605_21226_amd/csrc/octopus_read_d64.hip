#define OCTOPUS_D 64
#include "octopus_plans_read.inc"
