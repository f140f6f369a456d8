"""The same look at the kernels over the 4-bit cache (AMD assembly, compiled here; no GPU)."""
import re

import test_matrix_waits as T


def test_inline_instructions_of_the_kernel_of_many_rows_wait_for_matrix_results(tmp_path):
    T.test_inline_instructions_wait_for_matrix_results("attn_kv4_rows", tmp_path)


def test_the_other_cache_kernels_have_no_inline_instruction(tmp_path):
    for name in ("attn_kv4", "kv4_cache"):
        assert not any(inline and re.match(r"[vs]_|ds_|global_|buffer_", op)
                       for _kernel, code, _before in T._kernels(T._assembly(name, tmp_path)) for op, _args, inline in code), name
