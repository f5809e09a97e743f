"""An operator's bounded wait that expired is reported once, by the next call or by the status call. The
test program is the operators' C ABI with its internals in reach, linked with the library's other
objects; the word that a kernel would store to is written from the host."""

import pytest

from helpers import native_program, run_program

PROGRAM = r"""
#include "operators.cu"
#define EXPECT(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main(int argc, char**) {
  // no call yet: no word, nothing to report
  EXPECT(lipz_operator_status() == LIPZ_OK);
  if (argc < 2) return 0;
  float *x = nullptr, *scale = nullptr;
  unsigned char* q = nullptr;
  EXPECT(cudaMalloc(&x, 4096) == cudaSuccess && cudaMalloc(&scale, 256) == cudaSuccess);
  EXPECT(cudaMalloc(&q, 1024) == cudaSuccess && cudaMemset(x, 0, 4096) == cudaSuccess);
  lipz_quantize_rows_args a{};
  a.struct_size = sizeof a;
  a.groups = 1, a.rows = 4, a.dim = 256;
  a.x = {x, 0, 256, LIPZ_FP32, 0};
  a.q = {q, 0, 256, LIPZ_E4M3, 0};
  a.scale = {scale, 0};
  EXPECT(lipz_quantize_rows(&a, nullptr) == LIPZ_OK);
  int* word = ops::timeout_word();
  EXPECT(word && *word == 0);
  *word = 3;
  EXPECT(lipz_operator_status() == LIPZ_ERR_TIMEOUT);
  EXPECT(lipz_operator_error()[0] != 0);
  EXPECT(lipz_operator_status() == LIPZ_OK);
  *word = 4;
  EXPECT(lipz_quantize_rows(&a, nullptr) == LIPZ_ERR_TIMEOUT);
  EXPECT(lipz_quantize_rows(&a, nullptr) == LIPZ_OK);
  EXPECT(cudaDeviceSynchronize() == cudaSuccess);
  EXPECT(lipz_operator_status() == LIPZ_OK);
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return native_program(tmp_path_factory, "operator_status", PROGRAM, replaces=("operators.cu",))


def test_nothing_is_reported_before_a_call(program):
    run_program(program)


@pytest.mark.gpu
def test_an_expired_wait_is_reported_once(program):
    run_program(program, "gpu")
