#define CODE_BITS 2
#include "codes_product_inst.hpp"
