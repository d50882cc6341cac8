"""How the language side's attention is compiled."""
from paper_2609_31551_amd import build


def test_files_whose_calls_say_what_a_nan_does_are_built_to_honour_it():
    for name in ("prompt_attention.hip", "kv8_attention.hip", "kv8_cache.hip"):
        flags = build.FLAGS + build.FILE_FLAGS.get(name, [])
        assert not [f for f in flags if "honor-nans" in f or "finite-math" in f or "fast-math" in f or f == "-Ofast"], name
