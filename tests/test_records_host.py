"""What emr_device_error makes of several records of waits that gave up, compiled for the host: none is lost where two hold a number."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
#include <cstdio>
#include "%s/paper_2608_27612_gb300/csrc/emr_records.h"
struct Record {
  int held;
  emr_status status;
  int reads;
  emr_status operator()(int32_t* code) {
    reads++;
    if (status == EMR_OK) *code = held, held = 0;
    return status;
  }
};
static void ask(Record& a, Record& b) {
  int32_t code = -1;
  const int ok = emr::first_record([&](int32_t* c) { return a(c); }, [&](int32_t* c) { return b(c); }, &code);
  std::printf("%%d %%d %%d %%d\\n", ok, code, a.held, b.held);
}
int main() {
  Record a{7, EMR_OK, 0}, b{13, EMR_OK, 0}, bad{5, EMR_ERR_CUDA, 0};
  ask(a, b), ask(a, b), ask(a, b);
  ask(bad, b), ask(a, bad);
  a.held = 3;
  ask(a, bad);
  return 0;
}
"""


def test_one_record_after_the_other(tmp_path):
    source = tmp_path / "records.cpp"
    source.write_text(PROGRAM % ROOT)
    subprocess.run(["g++", "-std=c++17", "-o", str(tmp_path / "records"), str(source)], check=True, capture_output=True)
    lines = subprocess.run([str(tmp_path / "records")], check=True, capture_output=True, text=True).stdout.split("\n")
    ok, cuda = 0, 5
    assert lines[:3] == ["%d 7 0 13" % ok, "%d 13 0 0" % ok, "%d 0 0 0" % ok]     # the second is told by the second call
    assert lines[3:6] == ["%d -1 5 0" % cuda, "%d -1 0 5" % cuda, "%d 3 0 5" % ok]  # a failed read is reported, and tells nothing
