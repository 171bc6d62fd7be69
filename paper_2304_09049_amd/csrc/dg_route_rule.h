// Which kernel computes a router's logits, and the work buffer's size, by the call's sizes and the device's compute units alone: host code, free of the device's headers.
#pragma once

#include <stddef.h>
#include <stdint.h>

constexpr int DG_ROUTE_PARTS = 4;        // of K, where tiles of 16 tokens and 16 experts are fewer than the compute units

// By token and expert: one token a workgroup, or four.  By tiles of 16 x 16 tokens and experts, the same with K in parts, or of 32 x 32.
enum class DgRouteForm { One, Four, Tiles16, Parts16, Tiles32 };

inline int64_t dg_route_tiles(int64_t T, int64_t E, int side) { return (T + side - 1) / side * ((E + side - 1) / side); }
// The few-token kernel reads the router once for four tokens and takes sums one by one: it is the faster one to some 2500 sums (us with the choice, its and the others' with K in parts:
// 64 x 5120 to 16 experts, router in binary32, 8.1 and 9.5, 128 tokens 9.8 and 9.6; 32 x 4096 to 64 7.9 and 8.5, 64 tokens 9.3 and 8.7; 64 x 1352 to 64 7.2 and 7.7; 64 x 2048 to 128 9.7 and 7.8).
inline bool dg_route_few(int64_t T, int64_t E) { return T == 1 || T * E <= 2560; }
// A tile's products by one compute unit bound what has fewer tiles than there are units, whatever the number of tokens: K in parts, one and four (128 x 4096 to 64 17.4 and 8.8, 512 x 5120 to 16 20.3 and
// 9.8, 256 x 2048 to 128 12.2 and 9.8, but 1024 x 1352 to 64, 256 tiles, 11.5 and 12.1).  (The work buffer's size goes by this, so it does not ask for the device.)
inline bool dg_route_in_parts(int64_t T, int64_t E) { return !dg_route_few(T, E) && dg_route_tiles(T, E, 16) <= 192; }

// Of the tiles the larger are the faster ones where every compute unit gets two (us, the smaller's and the larger's, before loads ran ahead: 2048 x 2048 to 128 32.6 and 35, 4096 x 2048 to 128 55 and 53,
// 6000 x 4096 to 64 80 and 96, 8192 x 2048 to 256 with a router in binary32 193 and 171).  What is in parts is so before that is asked: on a device of a few units both may hold.
inline DgRouteForm dg_route_form(int64_t T, int64_t E, int64_t K, int64_t units)
{
    if (T == 1) return DgRouteForm::One;
    if (dg_route_few(T, E)) return DgRouteForm::Four;
    if (dg_route_in_parts(T, E) && K >= 1024) return DgRouteForm::Parts16;
    return dg_route_tiles(T, E, 32) >= 2 * units ? DgRouteForm::Tiles32 : DgRouteForm::Tiles16;
}

// Logits in binary32, or the parts' sums in binary64, whichever a call of so many tokens or of fewer takes more for: a buffer for a program's largest batch suffices for its others.  (What is in parts is at most 192
// tiles, 1.5 MB of sums; the most tokens that may be are the last before a 193rd.)
inline size_t dg_route_work_bytes(int64_t T, int64_t E)
{
    const int64_t most = 192 / ((E + 15) / 16) * 16, parts = T < most ? T : most;
    const int64_t whole = T * E * (int64_t)sizeof(float), sums = dg_route_in_parts(parts, E) ? parts * E * DG_ROUTE_PARTS * (int64_t)sizeof(double) : 0;
    return (size_t)(whole > sums ? whole : sums);
}
