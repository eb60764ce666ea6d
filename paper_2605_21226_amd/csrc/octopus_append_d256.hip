#define OCTOPUS_D 256
#include "octopus_plans_append.inc"
