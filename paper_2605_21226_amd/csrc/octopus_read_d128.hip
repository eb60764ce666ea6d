#define OCTOPUS_D 128
#include "octopus_plans_read.inc"
