// Every kernel of the library, in one translation unit: the library carries one device image.
#include "kernels.hip"
#include "differential.hip"
#include "beam.hip"
#include "pagecopy.hip"
#include "rotary.hip"
#include "slots.hip"
