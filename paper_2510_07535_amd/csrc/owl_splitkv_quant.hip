// The split-KV pass (owl_splitkv.h) for caches of 8-bit blocks, queries in 16 bits.
#include "owl_splitkv.h"

namespace owl {

static const Variant kQuantVariants[] = {
    OWL_VARIANTS_16BIT(OWL_BF16, __bf16, 128, false, true),
    OWL_VARIANTS_16BIT(OWL_BF16, __bf16, 64, false, true),
    OWL_VARIANTS_16BIT(OWL_F16, _Float16, 128, false, true),
    OWL_VARIANTS_16BIT(OWL_F16, _Float16, 64, false, true),
};

VariantList quant_variants() { return VariantList{kQuantVariants, (int)(sizeof kQuantVariants / sizeof kQuantVariants[0])}; }

}  // namespace owl
