"""Which cluster size the token scores launch with, on the host: the CUDA calls are stood in for by a record of the launches and a
device on which clusters of 16 do or do not find room."""
import os
import subprocess

import pytest

from paper_2609_01024_b200 import build

SOURCE = r"""
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

static int fit_16, asked, cluster, status_of_question;
static cudaError_t fake_device(int *d) { *d = 0; return cudaSuccess; }
template <typename F> cudaError_t fake_attribute(F *, cudaFuncAttribute, int) { return cudaSuccess; }
template <typename F> cudaError_t fake_question(int *n, F *, const cudaLaunchConfig_t *cfg) {
  ++asked;
  *n = cfg->attrs[cfg->numAttrs - 1].val.clusterDim.x <= 8 ? 18 : fit_16;
  return (cudaError_t)status_of_question;
}
template <typename F, typename... A> cudaError_t fake_launch(const cudaLaunchConfig_t *cfg, F *, A...) {
  cluster = 1;
  for (unsigned i = 0; i < cfg->numAttrs; ++i)
    if (cfg->attrs[i].id == cudaLaunchAttributeClusterDimension) cluster = (int)cfg->attrs[i].val.clusterDim.x;
  if (cfg->gridDim.x % cluster) return cudaErrorInvalidConfiguration;
  return cluster > 8 && !fit_16 ? cudaErrorInvalidClusterSize : cudaSuccess;
}
static cudaError_t fake_error() { return cudaSuccess; }
#define cudaGetDevice fake_device
#define cudaFuncSetAttribute fake_attribute
#define cudaOccupancyMaxActiveClusters fake_question
#define cudaLaunchKernelEx fake_launch
#define cudaGetLastError fake_error
#include "scores.cu"

namespace pcomoe {
void count_launch(int) {}
pcomoe_status current_sms(int *sms) { *sms = 148; return PCOMOE_OK; }
}

int main(int argc, char **argv) {
  fit_16 = atoi(argv[1]);
  status_of_question = atoi(argv[2]);
  for (int T : {1, 1, 4, 30, 60})
    for (int dtype : {0, 1}) {
      float lp[1];
      const int st = pcomoe_token_logprobs(dtype, T, 128000, (void *)4096, 128000, nullptr, 0, nullptr, lp, nullptr, nullptr, nullptr);
      printf("%d %d %d\n", T, st, cluster);
    }
  printf("asked %d\n", asked);
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("clusters")
    src, exe = d / "clusters.cu", d / "clusters"
    src.write_text(SOURCE)
    subprocess.run([build.NVCC, *build.FLAGS, str(src), "-o", str(exe), "-lcudart"], check=True, capture_output=True)
    return str(exe)


@pytest.mark.parametrize("fit,answer,largest", [(8, 0, 16), (0, 0, 8), (0, 1, 8)], ids=["fits", "no room", "question fails"])
def test_a_smaller_cluster_where_16_find_no_room(program, fit, answer, largest):
    env = dict(os.environ, LD_LIBRARY_PATH="/usr/local/cuda/lib64:" + os.environ.get("LD_LIBRARY_PATH", ""))
    out = subprocess.run([program, str(fit), str(answer)], env=env, check=True, capture_output=True, text=True).stdout.split("\n")
    rows = [tuple(map(int, x.split())) for x in out if x and not x.startswith("asked")]
    assert [st for _, st, _ in rows] == [0] * len(rows), rows                        # no call is refused
    assert [c for t, _, c in rows if t == 1] == [largest] * 4 and [c for t, _, c in rows if t == 60] == [4] * 2, rows
    assert int(out[-2].split()[1]) == 2                                              # once for each type
