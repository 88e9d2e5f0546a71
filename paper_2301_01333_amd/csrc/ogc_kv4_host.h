// Host-side checks shared by the operators of the 4-bit cache.
#ifndef OGC_KV4_HOST_H
#define OGC_KV4_HOST_H

#include "ogc_decoder.h"

ogc_status ogc_kv4_check(const ogc_kv4_desc* cache);

#endif
