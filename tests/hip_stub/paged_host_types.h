// Vector types that the paged cache's host code names, for the CPU build (included in front of everything).
#pragma once
struct int2 { int x, y; };
struct float2 { float x, y; };
