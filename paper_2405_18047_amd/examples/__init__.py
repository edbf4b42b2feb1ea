"""Small programs that put the library's operations together."""
