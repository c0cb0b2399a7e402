// C interface of the places on the stack of free pages for the CPU tests.
#include "../../paper_2605_27740_amd/csrc/place_plan.hpp"

extern "C" int stack_place(int size, long long before, int capacity) { return unique::stack_place(size, before, capacity); }
extern "C" int stack_has(int place, int i, int capacity) { return unique::stack_has(place, i, capacity); }
