"""Results that are written past the last-level cache, whole lines at a time, and
beside the cases that are not: the same values either way."""
import os
import re
import subprocess

import pytest

from tests.gpu_util import require_gpu


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{instance: assembly} of the product's tile kernels."""
    from paper_1904_05347_amd import build
    src = os.path.join(build.CSRC, "pk_gemm_i8.hip")
    out = str(tmp_path_factory.mktemp("asm") / "gemm_i8.s")
    subprocess.run([build.HIPCC] + [f for f in build.CFLAGS if f != "-fPIC"] + ["--cuda-device-only", "-S", src, "-o", out],
                   check=True, capture_output=True)
    with open(out) as fh:
        text = fh.read()
    found = {m.group(1): m.group(0) for m in
             re.finditer(r"^\S*gemm_i8_tile_kernelI(\w+?)EEEv\S*:.*?s_endpgm", text, re.S | re.M)}
    assert len(found) >= 3 * 14
    return found


def test_stores_past_the_cache_are_compiled(kernels):
    """The compiler may make one plain store of two branches that differ in the hint
    alone: the 16-byte stores of the large tiles come in both kinds."""
    large = {n: k for n, k in kernels.items() if re.match(r"\w+?Li(128|256)ELi(128|256)E", n)}
    assert len(large) >= 3 * 5
    for name, k in large.items():
        stores = re.findall(r"global_store_dwordx4 .*", k)
        past = [s for s in stores if s.rstrip().endswith(" nt")]
        assert past and len(past) < len(stores), name


def test_the_loop_waits_for_copies_only_where_it_says_so(kernels):
    """Where operands are copied straight to LDS, the loop over K-blocks has no wait
    for memory beside those written out: one of the compiler's would be for every
    copy in flight."""
    seen = 0
    for name, k in kernels.items():
        if not name.endswith("Lb1"):
            continue
        for _, body in re.findall(r"^(\.LBB\d+_\d+):[^\n]*Inner Loop Header[^\n]*\n(.*?)s_cbranch_\w+ \1\n", k, re.S | re.M):
            if "v_mfma" in body:
                seen += 1
                assert "vmcnt" not in re.sub(r";;#ASMSTART.*?;;#ASMEND", "", body, flags=re.S), name
    assert seen >= 3 * 8


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,ld,offset", [
    (10000, 8192, 333, 8192, 0),     # past it, whole tiles of columns
    (10000, 8190, 333, 8192, 0),     # past it, the last columns one by one
    (9999, 8190, 333, 8190, 0),      # rows off the lines
    (9999, 8190, 333, 8192, 1),      # a first column off the lines
    (5000, 8192, 333, 8192, 0),      # small enough to stay
    (70000, 500, 2000, 512, 0),      # many rows of few columns
])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_large_results(M, N, K, ld, offset, kind):
    torch, pk = require_gpu()
    T = getattr(torch, kind)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a = torch.randint(-128, 128, (M, (K + 3) // 4 * 4), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    b = torch.randint(-128, 128, (N, (K + 3) // 4 * 4), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    sa = torch.full((M,), 2.0 ** -9, device="cuda")   # powers of two: the fp32 value is exact
    sb = torch.full((N,), 2.0 ** -6, device="cuda")
    wide = torch.full((M, ld + 128 // (4 if kind == "float32" else 2)), 7.0, device="cuda", dtype=T)
    out = wide[:, offset:offset + N]
    pk.gemm_i8(a, b, sa, sb, out=out)
    bt = b.double().t().contiguous()
    for m in range(0, M, 4096):
        want = ((a[m:m + 4096].double() @ bt) * 2.0 ** -15).float().to(T)
        assert torch.equal(out[m:m + 4096], want), m
    assert (wide[:, :offset] == 7).all() and (wide[:, offset + N:] == 7).all()
