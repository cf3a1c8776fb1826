#define CODE_BITS 6
#include "codes_product_inst.hpp"
