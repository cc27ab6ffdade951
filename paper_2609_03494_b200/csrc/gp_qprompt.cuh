// Host side of the attention kernel for many rows of a sequence (gp_qprompt.cu), as gp_qcache_attention calls it.
#pragma once
#include "gp_qattn.cuh"

struct QpPlan { int blocks; };
QpPlan qp_plan(const QcDev& c, int G);
size_t qp_bytes(const QpPlan& p, int d);
int qp_launch(const QcDev& c, QtArgs a, const QpPlan& p, int d, void* work, cudaStream_t s);
