#define CODE_BITS 1
#include "codes_product_inst.hpp"
