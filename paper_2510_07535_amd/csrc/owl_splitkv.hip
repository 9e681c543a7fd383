// The split-KV pass (owl_splitkv.h) for caches of 16- and 32-bit numbers, and the list of all its variants.
#include "owl_splitkv.h"

namespace owl {

static const Variant kVariants[] = {
    OWL_VARIANTS_16BIT(OWL_BF16, __bf16, 128, false, false),
    OWL_VARIANTS_16BIT(OWL_BF16, __bf16, 64, false, false),
    OWL_VARIANTS_16BIT(OWL_F16, _Float16, 128, false, false),
    OWL_VARIANTS_16BIT(OWL_F16, _Float16, 64, false, false),
    make_variant<float, 64, 1, 8, 1, false, false>(OWL_F32),
    make_variant<float, 128, 1, 8, 1, false, false>(OWL_F32),
    // copies with the per-workgroup timeline hook: the benchmark's type and head size only
    OWL_VARIANTS_16BIT(OWL_BF16, __bf16, 128, true, false),
};
constexpr int kCount = sizeof kVariants / sizeof kVariants[0];

const Variant *find_variant(int dtype, int D, int tpw, int wr, int wk, bool timeline, bool quant)
{
    const VariantList quantised = quant_variants();
    const Variant *list = quant ? quantised.first : kVariants;
    for (int i = 0; i < (quant ? quantised.count : kCount); ++i) {
        const Variant &v = list[i];
        if (v.dtype == dtype && v.D == D && v.tpw == tpw && v.wr == wr && v.wk == wk && v.timeline == timeline) return &v;
    }
    return nullptr;
}

int variant_index(const Variant *v)
{
    if (!v) return -1;
    return static_cast<int>(v->quant ? kCount + (v - quant_variants().first) : v - kVariants);
}

}  // namespace owl
