// overlap.h for test_overlap.py: areas as {address, bytes of an element, elements of a piece, three walks of {pieces, step}}.
#include "overlap.h"

using namespace reform;

static Area area(const int64_t *x)
{
    return area_of((const void *)(uintptr_t)x[0], x[1], x[2], {{x[3], x[4]}, {x[5], x[6]}, {x[7], x[8]}});
}

extern "C" int overlap_meet(const int64_t *a, const int64_t *b) { return areas_meet(area(a), area(b)); }
extern "C" int overlap_empty(const int64_t *a) { return area(a).end == 0; }
