// The checks and the device form of an sd_rules, shared by sd_logits_rules and sd_set_rules (host only).
#pragma once
#include "sdfp_rules.hip.h"
#include "sdfp.h"

#include <cmath>

namespace sdfp {

inline bool rules_ok(const sd_rules& r) {
    if (!std::isfinite(r.repetition) || !(r.repetition > 0.f) || !std::isfinite(r.presence) || !std::isfinite(r.frequency)) return false;
    if (((uintptr_t)r.bias | (uintptr_t)r.allowed) & 3) return false;
    return !r.allowed || r.n_masks >= 1;
}
inline RuleSet rule_set(const sd_rules& r) {
    return RuleSet{r.repetition, r.presence, r.frequency, r.bias, r.allowed, r.allowed ? r.n_masks : 0};
}

}  // namespace sdfp
