"""CPU checks of the training operators' host side: sizes and what the Python
wrappers do around the kernels."""
import os
import subprocess

from paper_2609_15160_amd import tlf

INC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def test_kept_bytes_match_the_header(tmp_path):
    """18 bits for each of two values in bf16, 32 in float32, of whole 16 rows."""
    cases = [(t, rows, f) for t in (tlf.DTYPE_F32, tlf.DTYPE_BF16) for rows in (0, 1, 15, 16, 17, 66000, 2 ** 29)
             for f in (64, 192, 16384)]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "tlf.h"\nint main(void){' + "".join(
        f'printf("%zu\\n",tlf_ffn_kept_bytes({t},{rows},{f}));' for t, rows, f in cases) + "return 0;}")
    subprocess.check_call(["gcc", "-std=c99", "-I", INC, str(src), "-o", str(tmp_path / "t")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    for n, (t, rows, f) in zip(got, cases):
        bits = (rows + 15) // 16 * 16 * f * 2 * (18 if t == tlf.DTYPE_BF16 else 32)
        assert n == tlf.ffn_kept_bytes(t, rows, f) == bits // 8 and n % 16 == 0
