"""The structures of a drafted decoder step of include/ilpm.h as packed bytes, for calls of the C ABI from the tests."""
import struct

APPEND = struct.Struct("@PPPPPPPiiiiif")    # ilpm_append_options
TREE = struct.Struct("@Pqffiiii")           # ilpm_tree_options
VERIFY = struct.Struct("@PPPPqqqqPPPPiiii")  # ilpm_verify_args
