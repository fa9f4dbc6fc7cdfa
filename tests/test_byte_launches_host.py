"""Which kernels the gradients of linear layers on rows of 8 bits, and blocks that multiply such rows, go to, on the CPU: the launches that a call
asks a stand-in for the HIP runtime for (host_hip.py).  Addresses stand for buffers of any size and are never read."""
import os
import subprocess

import pytest

from host_hip import LIB, SOURCE, calls, compile_runtime
from paper_2411_12780_amd import synth

MAIN = r"""
struct Rows { void* p; int64_t ld; };
struct ByteRows { void *q, *e; int64_t ld; };
struct Config { uint32_t size; int32_t precision, rows, in, out, activation; };
int main(int, char** argv) {
  lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
  if (!lib) { std::fprintf(stderr, "%s\n", dlerror()); return 2; }
  Config c{sizeof(Config), 0, 0, 0, 0, 0};
  long ldy, ldx, ldg;
  int dx, dw, forward;
  while (std::cin >> forward >> c.precision >> c.rows >> c.in >> c.out >> ldy >> ldx >> ldg >> dx >> dw) {
    auto at = [](long i) { return (void*)(intptr_t)(i << 44); };
    const int64_t ld8 = (c.in + 15) / 16 * 16;
    ByteRows x{at(1), at(2), ld8}, w{at(3), at(4), ld8};
    Rows gy{at(5), ldy}, gx{at(6), ldx}, gate{at(7), ldg};
    size_t need = 0;
    ok(call("ppll_byte_linear_workspace_bytes", &c, &need), "size");
    std::printf("== %zu\n", need);
    logging = true;
    if (forward) {       // with GELU and its slope, or with a residual (gate), or neither
      c.activation = forward == 2 ? 3 : 0;
      ok(call("ppll_byte_linear_forward", &c, &x, &w, at(9), ldg ? &gate : (Rows*)nullptr, &gy, forward == 2 ? &gx : (Rows*)nullptr, (void*)nullptr), "forward");
      logging = false;
      continue;
    }
    ok(call("ppll_byte_linear_backward", &c, dw ? &x : (ByteRows*)nullptr, dx ? &w : (ByteRows*)nullptr, &gy, dx && ldg ? &gate : (Rows*)nullptr,
            dx ? &gx : (Rows*)nullptr, dw ? at(8) : nullptr, dw ? at(9) : nullptr, at(10), need, (void*)nullptr), "backward");
    logging = false;
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    directory = str(tmp_path_factory.mktemp("linear"))
    src, exe = os.path.join(directory, "b.cpp"), os.path.join(directory, "b")
    with open(src, "w") as f:
        f.write(SOURCE.split("int main(")[0] + MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-rdynamic", src, "-o", exe, "-ldl"], check=True)

    def run(*line):
        r = subprocess.run([exe, LIB], input=" ".join(map(str, line)), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        launches = [(tuple(map(int, f[2:5])), int(f[5]), f[7]) for f in (line.split() for line in r.stdout.splitlines()) if f[0] == "launch"]
        for grid, threads, name in launches:       # what a launch holds
            assert grid[1] < 65536 and grid[2] < 65536 and grid[0] * threads < 1 << 32, (grid, threads, name)
        return [name for _, _, name in launches]
    return run


@pytest.fixture(scope="module")
def backward(program):
    def run(rows, n_in, n_out, room_y=0, room_x=0, gate=False, dx=True, dw=True, precision=1):
        return program(0, precision, rows, n_in, n_out, n_out + room_y, n_in + room_x, n_in if gate else 0, int(dx), int(dw))
    return run


@pytest.fixture(scope="module")
def forward(program):
    def run(rows, n_in, n_out, gelu=False, residual=False, precision=1):
        return program(2 if gelu else 1, precision, rows, n_in, n_out, n_out, n_out, n_out if residual else 0, 0, 0)
    return run


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    exe = compile_runtime(str(tmp_path_factory.mktemp("runtime")))
    return lambda workloads, *what: calls(exe, workloads, *what)


@pytest.mark.parametrize("precision", [0, 1])
@pytest.mark.parametrize("rows,n_in", [(1 << 30, 16), (1 << 30, 112), ((1 << 30) - 1000, 128), (1 << 29, 256), (1 << 28, 512)])
@pytest.mark.parametrize("end", [dict(), dict(gelu=True), dict(residual=True)], ids=str)
def test_a_product_of_very_many_rows_fits_a_launch(forward, precision, rows, n_in, end):
    # up to 2^23 tiles of 128 x 128, on which a workgroup of the kernel with copying waves has 512 threads
    for n_out in (8, 128):
        names = forward(rows, n_in, n_out, precision=precision, **end)
        assert len(names) == 1 and "byte_linear" in names[0]


# both sides of 2^28 elements of dX (where the bf16 kernels end), by columns, by rows' distance, by rows alone
FAR = [dict(rows=65535, n_in=4096, n_out=4096), dict(rows=65536, n_in=4096, n_out=4096), dict(rows=65536, n_in=6144, n_out=1536),
       dict(rows=100864, n_in=2816, n_out=768), dict(rows=131071, n_in=2048, n_out=512), dict(rows=200000, n_in=2048, n_out=512),
       dict(rows=5000000, n_in=64, n_out=64), dict(rows=8192, n_in=1536, n_out=1536, room_x=64000), dict(rows=512, n_in=2048, n_out=2048, room_x=(1 << 19) + 8),
       dict(rows=512, n_in=8192, n_out=8192, room_x=(1 << 19) + 8), dict(rows=600, n_in=18000, n_out=20000), dict(rows=1024, n_in=4096, n_out=4096, room_y=(1 << 19) + 8)]


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("dw", [False, True])
@pytest.mark.parametrize("size", FAR, ids=str)
def test_no_gradient_is_left_to_the_kernel_without_matrix_instructions(backward, size, dw, gate):
    names = backward(**size, dw=dw, gate=gate)
    assert names and not any("gemm_generic" in n or "gemm_f32" in n for n in names), names


def test_dx_of_many_elements_in_stretches_of_rows(backward):
    # as one product at 65535 x 4096, as two at 65536, on the kernel that reads the bytes where a stretch would be of few rows
    products = lambda **k: [n for n in backward(**k, dw=False) if "gemm" in n]  # noqa: E731
    assert len(products(rows=65535, n_in=4096, n_out=4096)) == 1
    assert len(products(rows=65536, n_in=4096, n_out=4096)) == 2
    one, two = (products(rows=r, n_in=4096, n_out=4096) for r in (32768, 65536))
    assert two == 2 * one
    for far in (dict(room_x=(1 << 19) + 8), dict(room_y=(1 << 20) - 2048)):
        names = backward(rows=512 + 2048 * ("room_y" in far), n_in=2048, n_out=2048, dw=False, **far)
        assert names and all("byte_grad" in n for n in names), names
    assert any("byte_grad_kernel" in n for n in backward(rows=600, n_in=18000, n_out=20000))      # dW of 2^28 elements and more


def vit(byte_products, depth, aux_depth, batch=16, dim=128, precision=synth.BF16, **more):
    return synth.workload("vit_stage_act_bf16", tokens=17, dim=dim, heads=dim // 64, mlp_dim=4 * dim, batch=batch, precision=precision, depth=depth, aux_depth=aux_depth,
                          byte_products=byte_products, **more)


@pytest.mark.parametrize("precision", [synth.FP32, synth.BF16])
@pytest.mark.parametrize("depth,aux_depth,layers", [(1, 0, 1), (1, 1, 1), (2, 1, 2), (1, 2, 2), (3, 3, 5)])
def test_every_layer_but_the_pruned_one_multiplies_bytes(runtime, precision, depth, aux_depth, layers):
    made = lambda bytes_: [[c[5] for c in call if c[0] == "launch"] for call in runtime([vit(bytes_, depth, aux_depth, precision=precision)], "step", "eval", "eval_noalloc")]  # noqa: E731
    count = lambda names, *parts: sum(any(p in n for p in parts) for n in names)  # noqa: E731
    for i, names in enumerate(made(1)):
        assert count(names, "byte_linear") == 4 * layers
        assert count(names, "byte_rows_pack_columns") == 4 * layers
        assert count(names, "byte_rows_pack_kernel", "byte_rows_pack_long") == 4 * layers
        assert count(names, "byte_grad_kernel", "byte_rows_values") == (4 * layers if i == 0 else 0)
    for names in made(0):
        assert not count(names, "byte_")


@pytest.mark.parametrize("batch,call", [(50, "step"), (50, "batch"), (4, "batch"), (4, "eval")])
def test_a_launch_asks_for_the_device_less_than_once(runtime, batch, call):
    wl = dict(vit(1, 1, 1, batch=batch, dim=1024), tokens=65)
    (made,) = runtime([wl] * (2 if call == "batch" else 1), call)
    asked, launches = (sum(c[0] == kind for c in made) for kind in ("device", "launch"))
    assert asked < launches, (asked, launches)


def test_products_of_a_pipeline_leave_the_units_to_each_other(runtime):
    # dX of the first MLP layer, 3250 rows of 1024 from 4096 channels, in values: alone on 208 tiles with copying waves, one a unit (512 threads, four stages
    # of 64 k); in a pipeline on what it would be without rows of 8 bits
    copying = lambda made: [c for c in made if c[0] == "launch" and "gemm_pipe" in c[5] and "ELi2ELi2ELi2ELi4ELi64E" in c[5]]  # noqa: E731
    wl = dict(vit(1, 1, 0, batch=50, dim=1024), tokens=65)
    alone, batch = runtime([wl], "step")[0], runtime([wl, wl], "batch")[0]
    assert any("byte_rows_values" in c[5] for c in alone if c[0] == "launch")
    assert copying(alone) and not copying(batch)
