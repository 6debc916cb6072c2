/* Element types of the entry points that take more than one (mi355lp.h, mi355gn.h, mi355q4.h, mi355sm.h, mi355i8.h). */
#ifndef MI355DTYPE_H
#define MI355DTYPE_H

typedef enum {
  MI355_F32 = 0,
  MI355_F16 = 1,  /* IEEE binary16 */
  MI355_BF16 = 2,
  MI355_F64 = 3   /* mi355gn.h only */
} mi355_dtype_t;

#endif
