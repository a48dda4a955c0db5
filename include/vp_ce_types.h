/* vp_ce_types.h -- element types in calls that accept more than one (layer_norm.h, muon.h). */
#ifndef VP_CE_TYPES_H_
#define VP_CE_TYPES_H_

enum { VPCE_BF16 = 0, VPCE_F16 = 1, VPCE_F32 = 2 };

#endif /* VP_CE_TYPES_H_ */
