// The order in which a product's stages move through LDS (host and device; no HIP, so that a
// host program can follow it load by load).
#pragma once

#include <cstdint>
#include <type_traits>

namespace gl {

// The contraction goes by halves of a stage.  An operand along it lies in a ring of whole
// stages, one down it (DOWN) in a ring of halves.  Half h is piece h of a ring of halves, and
// half h & 1 of piece h / 2 of one of stages.  LA, LB: direct loads a wave makes for a piece;
// PA, PB: a piece's bytes.
constexpr int product_ring_depth(bool down, bool other_down) {
  return down ? (other_down ? 5 : 4) : other_down ? 3 : 2;
}

template <bool DOWN_A, bool DOWN_B, int LA, int LB, uint32_t PA, uint32_t PB>
struct ProductRing {
  static constexpr bool HA = DOWN_A, HB = DOWN_B;  // by halves
  static constexpr int RA = product_ring_depth(HA, HB), RB = product_ring_depth(HB, HA);
  // Loads that may be under way while half h + 1 must have landed: those issued after its own.
  // Each turn issues the stages' (odd turns) and then the halves'.
  //   halves: h + 1's went out in turn h + 1 - ring; the ring - 2 turns up to h - 1 follow, of
  //     which half are odd (rounded up after an even h, as h - 1 is odd)
  //   stages: that of h + 1 (h odd) in turn h + 2 - 2 ring; 2 ring - 2 turns' halves follow,
  //     its own turn's among them, and ring - 2 stages
  static constexpr int per_stage = (HA ? 0 : LA) + (HB ? 0 : LB), per_half = (HA ? LA : 0) + (HB ? LB : 0);
  static constexpr int rh = HA ? RA : RB, rs = HA ? RB : RA;
  static constexpr int by_half_even = (rh - 2) * per_half + (rh - 1) / 2 * per_stage;
  static constexpr int by_half_odd = (rh - 2) * per_half + (rh - 2) / 2 * per_stage;
  static constexpr int by_stage = (rs - 2) * per_stage + (2 * rs - 2) * per_half;
  static constexpr int after_even = by_half_even;
  static constexpr int after_odd =
      HA && HB ? by_half_odd : HA || HB ? (by_half_odd < by_stage ? by_half_odd : by_stage) : by_stage;
  static constexpr int LAST = 2 * (RA > RB ? RA : RB);  // turns before the last whose loads all go out

  static constexpr uint32_t next(uint32_t at, uint32_t piece, int ring) {
    return at + piece == piece * (uint32_t)ring ? 0u : at + piece;
  }

  // Halves h0 .. h1 (even both).
  //   load_a(piece, at), load_b: a piece's loads to that place in its ring
  //   wait(N): all but the last N loads have landed, the reads before are done, in every wave;
  //     drain: all have landed
  //   read(set, a, b): half `set` (0 or 1) of its stage, or the half, that lies at a and b, to
  //     the registers of that set
  //   multiply(set): those registers' products
  // Once every wave has half h in registers, a piece that it was the last of is filled with
  // the one that comes a ring later.
  template <class LoadA, class LoadB, class Wait, class Drain, class Read, class Multiply>
  __attribute__((always_inline)) static constexpr void run(int h0, int h1, const LoadA& load_a, const LoadB& load_b,
                                                           const Wait& wait, const Drain& drain, const Read& read,
                                                           const Multiply& multiply) {
    using std::integral_constant;
    constexpr integral_constant<int, 0> first{};
    constexpr integral_constant<int, 1> second{};
    if (h0 >= h1) return;
    uint32_t pa = 0, pb = 0;  // where half h's pieces lie in the rings
    // after half h (odd: of its stage)
    auto fill = [&](int h, bool odd) {
      if (!HA && odd && 2 * ((h >> 1) + RA) < h1) load_a((h >> 1) + RA, pa);
      if (!HB && odd && 2 * ((h >> 1) + RB) < h1) load_b((h >> 1) + RB, pb);
      if (HA && h + RA < h1) load_a(h + RA, pa);
      if (HB && h + RB < h1) load_b(h + RB, pb);
    };
    // the rings' first filling, in the order of the turns that would have made it
#pragma unroll
    for (int o = 2 - LAST; o <= 0; ++o) {  // the turn before half h0 + o
      const bool odd = (o & 1) == 0;
      if (!HA && odd && o / 2 - 1 + RA >= 0 && h0 + 2 * (o / 2 - 1 + RA) < h1)
        load_a(h0 / 2 + o / 2 - 1 + RA, (o / 2 - 1 + RA) * PA);
      if (!HB && odd && o / 2 - 1 + RB >= 0 && h0 + 2 * (o / 2 - 1 + RB) < h1)
        load_b(h0 / 2 + o / 2 - 1 + RB, (o / 2 - 1 + RB) * PB);
      if (HA && o - 1 + RA >= 0 && h0 + o - 1 + RA < h1) load_a(h0 + o - 1 + RA, (o - 1 + RA) * PA);
      if (HB && o - 1 + RB >= 0 && h0 + o - 1 + RB < h1) load_b(h0 + o - 1 + RB, (o - 1 + RB) * PB);
    }
    if (h0 + LAST < h1) wait(integral_constant<int, after_odd>{});
    else drain();
    read(first, 0u, 0u);
    for (int h = h0; h < h1; h += 2) {
      uint32_t qa = HA ? next(pa, PA, RA) : pa, qb = HB ? next(pb, PB, RB) : pb;
      if constexpr (HA || HB) {
        if (h + LAST < h1) wait(integral_constant<int, after_even>{});
        else drain();
        fill(h, false);
      }
      read(second, qa, qb);
      multiply(first);
      pa = qa, pb = qb;
      qa = next(pa, PA, RA), qb = next(pb, PB, RB);
      if (h + LAST < h1) wait(integral_constant<int, after_odd>{});
      else drain();
      fill(h + 1, true);
      // (after the last half too, of whatever lies there: behind a branch the compiler would
      // not know how many reads are under way, and wait for these before it multiplies)
      read(first, qa, qb);
      multiply(second);
      pa = qa, pb = qb;
    }
  }
};

}  // namespace gl
