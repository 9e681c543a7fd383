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
    const VariantList list = !quant ? VariantList{kVariants, kCount} : wk == kWaves ? few_tile_variants() : quant_variants();
    for (int i = 0; i < list.count; ++i) {
        const Variant &v = list.first[i];
        if (v.dtype == dtype && v.D == D && v.tpw == tpw && v.wr == wr && v.wk == wk && v.timeline == timeline) return &v;
    }
    return nullptr;
}

int variant_index(const Variant *v)
{
    if (!v) return -1;
    if (!v->quant) return static_cast<int>(v - kVariants);
    const VariantList quant = quant_variants();
    return static_cast<int>(v->wk == kWaves ? kCount + quant.count + (v - few_tile_variants().first) : kCount + (v - quant.first));
}

}  // namespace owl
