#define OCTOPUS_D 256
#include "octopus_plans_read.inc"
