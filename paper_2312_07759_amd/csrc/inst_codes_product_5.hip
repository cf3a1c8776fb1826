#define CODE_BITS 5
#include "codes_product_inst.hpp"
