#define CODE_BITS 3
#include "codes_product_inst.hpp"
