#define OCTOPUS_D 64
#include "octopus_plans_append.inc"
