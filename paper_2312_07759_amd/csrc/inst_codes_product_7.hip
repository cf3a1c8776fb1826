#define CODE_BITS 7
#include "codes_product_inst.hpp"
