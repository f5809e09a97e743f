"""An expired wait is reported to the thread whose call it was, and to no other. The test program is the
operators' C ABI with its internals in reach; the words that kernels would store to are written from the host."""

import pytest

from helpers import native_program, run_program

PROGRAM = r"""
#include "operators.cu"
#include <set>
#include <thread>
#define EXPECT(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

static float *x, *scale;
static unsigned char* q;
static int call() {
  lipz_quantize_rows_args a{};
  a.struct_size = sizeof a;
  a.groups = 1, a.rows = 4, a.dim = 256;
  a.x = {x, 0, 256, LIPZ_FP32, 0};
  a.q = {q, 0, 256, LIPZ_E4M3, 0};
  a.scale = {scale, 0};
  return lipz_quantize_rows(&a, nullptr);
}

int main() {
  EXPECT(cudaMalloc(&x, 4096) == cudaSuccess && cudaMalloc(&scale, 256) == cudaSuccess);
  EXPECT(cudaMalloc(&q, 1024) == cudaSuccess && cudaMemset(x, 0, 4096) == cudaSuccess);
  EXPECT(call() == LIPZ_OK);
  int* mine = ops::timeout_word();
  EXPECT(mine && *mine == 0 && ops::timeout_word() == mine);
  *mine = 5;
  // another thread's calls go on, and what they report stays theirs
  int other = -1;
  std::thread([&] {
    other = [&] {
      EXPECT(lipz_operator_status() == LIPZ_OK && call() == LIPZ_OK);
      int* word = ops::timeout_word();
      EXPECT(word && word != mine && *word == 0);
      *word = 7;
      EXPECT(call() == LIPZ_ERR_TIMEOUT && strstr(lipz_operator_error(), "(7)"));
      EXPECT(call() == LIPZ_OK && lipz_operator_status() == LIPZ_OK);
      return 0;
    }();
  }).join();
  EXPECT(other == 0);
  EXPECT(lipz_operator_status() == LIPZ_ERR_TIMEOUT && strstr(lipz_operator_error(), "(5)"));
  EXPECT(lipz_operator_status() == LIPZ_OK && call() == LIPZ_OK);
  // a word of its own for each of many threads, clear
  std::set<int*> words{mine};
  bool clear = true;
  for (int i = 0; i < 2500; ++i)
    std::thread([&] {
      int* w = ops::timeout_word();
      clear = clear && w && *w == 0;
      words.insert(w);
      *w = 9;
    }).join();
  EXPECT(clear && words.size() == 2501);
  EXPECT(call() == LIPZ_OK && cudaDeviceSynchronize() == cudaSuccess && lipz_operator_status() == LIPZ_OK);
  return 0;
}
"""


@pytest.mark.gpu
def test_an_expired_wait_is_its_own_threads(tmp_path_factory):
    run_program(native_program(tmp_path_factory, "operator_threads", PROGRAM, replaces=("operators.cu",)))
