#define CODE_BITS 4
#include "codes_product_inst.hpp"
