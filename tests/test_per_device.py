"""Calls without a context run on whichever device is current, and a kernel's attributes belong to a device: what they set up
is set up once per device, not once per process."""
import os
import re
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1910_02120_b200", "csrc")
OPERATORS = ["layer_norm.cu", "norm_forward.cu", "norm_backward.cu", "norm_narrow.cu", "adamw.cu", "norm_rows.cuh"]

PROGRAM = r"""
#include "per_device.h"
#include <atomic>
#include <cstdio>
#include <thread>
#include <vector>

int main() {
  static ist::OncePerDevice<int> once;
  std::atomic<int> runs[80] = {};
  std::atomic<int> wrong{0};
  std::vector<std::thread> threads;
  for (int k = 0; k < 8; ++k)
    threads.emplace_back([&] {
      for (int round = 0; round < 100; ++round)
        for (int d = 0; d < 80; ++d)
          if (once.get(d, [&] { ++runs[d]; return 1000 + d; }) != 1000 + d) ++wrong;
    });
  for (auto& t : threads) t.join();
  for (int d = 0; d < 64; ++d) wrong += runs[d] != 1;
  for (int d = 64; d < 80; ++d) wrong += runs[d] != 800;      // beyond the table: every time
  wrong += once.get(-1, [] { return 7; }) != 7;
  std::printf("%d\n", (int)wrong);
  return wrong ? 1 : 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_every_device_has_its_own(tmp_path):
    source, program = tmp_path / "once.cpp", tmp_path / "once"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(source), "-o", str(program)], check=True)
    assert subprocess.run([str(program)], capture_output=True, text=True).stdout == "0\n"


@pytest.mark.parametrize("name", OPERATORS)
def test_kernel_attributes_are_set_per_device(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    assert "once_flag" not in text and "call_once" not in text
    for m in re.finditer(r"cudaFuncSetAttribute\(", text):
        assert "ready_here(once" in text[max(0, m.start() - 200):m.start()], name


@pytest.mark.gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_a_second_device():
    from paper_1910_02120_b200 import api
    results = []
    for device in ("cuda:0", "cuda:1"):                   # whichever is current, the tensors' device is used
        gen = torch.Generator().manual_seed(1)
        x, dy = torch.randn(512, 1024, generator=gen).bfloat16().to(device), torch.randn(512, 1024, generator=gen).to(device)
        y, mean, rstd = api.ist_layer_norm_forward(x)
        p = torch.ones(100000, device=device)
        opt = api.AdamW([p], state_bits=8, max_norm=1.0)
        opt.step([dy.view(-1)[:100000]])
        results.append([t.cpu() for t in (y, *api.ist_layer_norm_backward(dy, x, None, mean, rstd), p, *opt.state.values())])
    assert all(torch.equal(a, b) for a, b in zip(*results))
