"""The row operators' check of their buffers (rows.h), compiled for the host alone: an
output may be the buffer whose name it gives, wherever the two names lie in memory."""
import os
import subprocess

import pytest

from paper_1712_01537_amd import build

PROGRAM = r"""
#include <cstdio>
#include "rows.h"
namespace oc {
oc_status fail(oc_status s, const char*, ...) { return s; }
}  // namespace oc
int main() {
  char x[] = "x", again[] = "x", res[] = "res";
  char buf[64];
  const auto check = [&](const char* same, const char* name, char* at, size_t bytes) {
    const oc::Span s[] = {{"y", buf, 32, true, same}, {name, at, bytes, false, nullptr}};
    return (int)oc::check_spans("test", s);
  };
  std::printf("%d %d %d %d %d %d %d\n", check(x, again, buf, 32), check(x, x, buf, 32),
              check(x, res, buf, 32), check(nullptr, x, buf, 32), check(x, again, buf + 4, 32),
              check(x, again, buf, 16), check(x, again, buf + 32, 32));
}
"""


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
def test_in_place_outputs_are_known_by_name(tmp_path):
    src, exe = tmp_path / "spans.hip", tmp_path / "spans"
    src.write_text(PROGRAM)
    r = subprocess.run([build.HIPCC, "--offload-host-only", "-std=c++17", f"-I{build.INCLUDE}",
                        f"-I{build.CSRC}", str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert out.split() == ["0", "0", "1", "1", "1", "1", "0"]
