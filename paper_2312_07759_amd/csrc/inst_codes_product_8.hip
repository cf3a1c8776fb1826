#define CODE_BITS 8
#include "codes_product_inst.hpp"
